// Relative position bias by buckets and the gradient of its table (include/relative_bias.h).
//
// Both forms of the forward are a look-up in LDS beside a stream of stores (and of the base's loads).  The gradient is
// a sum by bucket: every lane adds into a column of LDS of its own, so that no two lanes meet, the order of the
// sums is fixed, and no two lanes of a wave share a bank.
#include <algorithm>
#include <cmath>

#include "common.h"
#include "kernels.h"
#include "vec.h"

namespace trimul {
namespace {

// The place of distance p_k - p_q in the look-up table, [0, 2 reach].
__device__ __forceinline__ int distance_index(int pk, int pq, int reach) {
    return min(max(__builtin_elementwise_sub_sat(pk, pq), -reach), reach) + reach;
}

// Lanes take eight neighbouring keys each, usually at eight neighbouring distances: with one place left free after
// every eight, the lanes of a wave read different banks.
__device__ __forceinline__ int skewed(int i) { return i + (i >> 3); }

__device__ __forceinline__ float table_value(const RelativeArgs& a, int row, int col) {
    const int64_t at = (int64_t)row * a.heads + col;
    return a.table_bf16 ? bf2f(static_cast<const bf16_t*>(a.table)[at]) : static_cast<const float*>(a.table)[at];
}

__device__ __forceinline__ int bucket_of(const RelativeArgs& a, int index) { return min((int)a.lut[index], a.buckets - 1); }

// Positions (and segments) of eight keys from j on; those behind the last are 0.
__device__ __forceinline__ void eight(const int32_t* p, int64_t j, int64_t n, int (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = j + i < n ? p[j + i] : 0;
}

// ---------------------------------------------------------------- bias [batch][heads][nq][nk]

// A work-group: `hb` heads, a.tx threads along the keys (eight each), 256 / a.tx rows at a time, a.loop times.
template <typename T, bool SEG, bool BASE>
__global__ __launch_bounds__(256) void k_relative_bias(const RelativeArgs a) {
    extern __shared__ float val[];
    int64_t at = blockIdx.x;
    const int cb = (int)(at % a.cblocks);
    at /= a.cblocks;
    const int rb = (int)(at % a.rblocks);
    at /= a.rblocks;
    const int hg = (int)(at % a.hblocks);
    const int64_t b = at / a.hblocks;
    const int h0 = hg * a.hb, nh = min(a.hb, a.heads - h0);
    const int entries = 2 * a.reach + 2, stride = skewed(entries) + 1;      // the last entry: another segment
    for (int e = threadIdx.x; e < entries * a.hb; e += 256) {
        const int i = e / a.hb, h = e - i * a.hb;                           // (hb is a power of two)
        if (h < nh) val[h * stride + skewed(i)] = table_value(a, i == entries - 1 ? a.buckets - 1 : bucket_of(a, i), h0 + h);
    }
    __syncthreads();
    const int tx = threadIdx.x & (a.tx - 1), ty = threadIdx.x / a.tx, rows = 256 / a.tx;
    const int64_t j = ((int64_t)cb * a.tx + tx) * 8;
    const int n = (int)min((int64_t)8, a.nk - j);
    if (n <= 0) return;
    int pk[8], sk[8];
    eight(a.pos_k + b * a.pos_k_batch, j, a.nk, pk);
    if constexpr (SEG) eight(a.seg_k + b * a.seg_k_batch, j, a.nk, sk);
    const T* base = static_cast<const T*>(a.base.data) + b * a.base.batch + h0 * a.base.head + j;
    T* out = static_cast<T*>(a.out.data) + b * a.out.batch + h0 * a.out.head + j;
    const int64_t r0 = (int64_t)rb * rows * a.loop, r1 = min(r0 + (int64_t)rows * a.loop, a.nq);
    for (int64_t r = r0 + ty; r < r1; r += rows) {
        const int pq = a.pos_q[b * a.pos_q_batch + r];
        int idx[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) idx[i] = distance_index(pk[i], pq, a.reach);
        if constexpr (SEG) {
            const int sq = a.seg_q[b * a.seg_q_batch + r];
#pragma unroll
            for (int i = 0; i < 8; ++i) idx[i] = sk[i] == sq ? idx[i] : entries - 1;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) idx[i] = skewed(idx[i]);
        for (int h = 0; h < nh; h += 4) {
            Vec<T, 8> v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (h + u >= nh) break;
                if constexpr (BASE) load_some(v[u], base + (h + u) * a.base.head + r * a.base.row, n, a.wide);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (h + u >= nh) break;
                const float* t = val + (h + u) * stride;
#pragma unroll
                for (int i = 0; i < 8; ++i) v[u].f[i] = BASE ? v[u].f[i] + t[idx[i]] : t[idx[i]];
                store_some(v[u], out + (h + u) * a.out.head + r * a.out.row, n, a.wide);
            }
        }
    }
}

// A work-group: one head of one entry, rows [split's share) on a.waves waves; 64 columns of LDS for each wave and bucket.
template <typename T, bool SEG>
__global__ __launch_bounds__(256) void k_relative_bias_backward(const RelativeArgs a) {
    extern __shared__ float val[];
    uint8_t* lut = reinterpret_cast<uint8_t*>(val + (size_t)a.waves * a.buckets * 64);
    int64_t at = blockIdx.x;
    const int split = (int)(at % a.splits);
    at /= a.splits;
    const int h = (int)(at % a.heads);
    const int64_t b = at / a.heads;
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, threads = a.waves * 64;
    for (int e = threadIdx.x; e <= 2 * a.reach; e += threads) lut[e] = (uint8_t)bucket_of(a, e);
    for (int e = threadIdx.x; e < a.waves * a.buckets * 64; e += threads) val[e] = 0.f;
    __syncthreads();
    float* acc = val + wave * a.buckets * 64 + lane;
    const int tx = lane & (a.tx - 1), ty = lane / a.tx, rows = 64 / a.tx, step = a.waves * rows;
    const int64_t per = (a.nq + a.splits - 1) / a.splits, r0 = split * per, r1 = min(r0 + per, a.nq);
    const T* from = static_cast<const T*>(a.out.data) + b * a.out.batch + h * a.out.head;
    const int32_t* pos_q = a.pos_q + b * a.pos_q_batch;
    const int32_t* seg_q = SEG ? a.seg_q + b * a.seg_q_batch : nullptr;
    for (int64_t j = (int64_t)tx * 8; j < a.nk; j += (int64_t)a.tx * 8) {
        const int n = (int)min((int64_t)8, a.nk - j);
        int pk[8], sk[8];
        eight(a.pos_k + b * a.pos_k_batch, j, a.nk, pk);
        if constexpr (SEG) eight(a.seg_k + b * a.seg_k_batch, j, a.nk, sk);
        auto add = [&](const Vec<T, 8>& v, int pq, int sq) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                int t = lut[distance_index(pk[i], pq, a.reach)];
                if constexpr (SEG) t = sk[i] == sq ? t : a.buckets - 1;
                atomicAdd(acc + t * 64, v.f[i]);        // (this lane's own: ds_add_f32 in the order of the program)
            }
        };
        int64_t r = r0 + wave * rows + ty;
        for (; r + 3 * step < r1; r += 4 * step) {
            Vec<T, 8> v[4];
            int pq[4], sq[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                load_some(v[u], from + (r + u * step) * a.out.row + j, n, a.wide);
                pq[u] = pos_q[r + u * step];
                sq[u] = SEG ? seg_q[r + u * step] : 0;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) add(v[u], pq[u], sq[u]);
        }
        for (; r < r1; r += step) {
            Vec<T, 8> v;
            load_some(v, from + r * a.out.row + j, n, a.wide);
            add(v, pos_q[r], SEG ? seg_q[r] : 0);
        }
    }
    __syncthreads();
    for (int t = threadIdx.x; t < a.buckets; t += threads) {
        double sum = 0;
        for (int w = 0; w < a.waves; ++w)
            for (int i = 0; i < 64; ++i) sum += val[(w * a.buckets + t) * 64 + ((i + t) & 63)];   // (each thread at a bank of its own)
        if (a.batch * a.splits == 1) a.dtable[(int64_t)t * a.heads + h] = (float)sum;
        else a.part[((b * a.splits + split) * a.heads + h) * a.buckets + t] = (float)sum;
    }
}

// dtable from `slots` partial tables [heads][buckets]: a lane for each value, a wave for every fourth slot.
__global__ __launch_bounds__(256) void k_relative_join(const RelativeArgs a, int64_t slots) {
    __shared__ double sums[4][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, n = a.heads * a.buckets;
    const int e = blockIdx.x * 64 + lane;
    double sum = 0;
    if (e < n)
        for (int64_t s = wave; s < slots; s += 4) sum += a.part[s * n + e];
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && e < n) {
        const int h = e / a.buckets, t = e - h * a.buckets;
        a.dtable[(int64_t)t * a.heads + h] = (float)(sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane]);
    }
}

__global__ __launch_bounds__(256) void k_relative_zero(float* p, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) p[i] = 0.f;
}

// ---------------------------------------------------------------- pair [nq][nk][channels]

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
    for (int e = threadIdx.x; e < a.buckets * width; e += 256) {
        const int t = e / width, c = e - t * width;
        val[e] = c < nc ? table_value(a, t, c0 + c) : 0.f;
    }
    for (int e = threadIdx.x; e <= 2 * a.reach; e += 256) lut[e] = (uint8_t)bucket_of(a, e);
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
        Vec<T, V> v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t j = j0 + u * pairs;
            if constexpr (BASE)
                if (j < a.nk) v[u].load(base + r * a.base.row + j * a.heads);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t j = j0 + u * pairs;
            int t = lut[distance_index(pk[u], pq, a.reach)];
            if constexpr (SEG) t = sk[u] == sq ? t : a.buckets - 1;
            Vec<float, V> w;
            w.load(val + t * width + lane * V);
#pragma unroll
            for (int i = 0; i < V; ++i) v[u].f[i] = BASE ? v[u].f[i] + w.f[i] : w.f[i];
            if (j < a.nk) v[u].store(out + r * a.out.row + j * a.heads);
        }
    }
}

// Sums by bucket over a tile of pairs.  A wave takes one pair at a time (a lane for V of its channels), so the bucket is
// one for the wave: the sum stays in registers while it does not change, and goes to the wave's own table in LDS
// when it does.
template <typename T, int V, bool SEG>
__global__ __launch_bounds__(256) void k_relative_pair_backward(const RelativeArgs a) {
    extern __shared__ float val[];
    constexpr int kAhead = 16;
    const int table = a.buckets * 64 * V;
    uint32_t* touched = reinterpret_cast<uint32_t*>(val + (size_t)a.waves * table);
    uint8_t* lut = reinterpret_cast<uint8_t*>(touched + 8);
    int64_t at = blockIdx.x;
    const int cb = (int)(at % a.hblocks);
    at /= a.hblocks;
    const int64_t tile = at;
    const int64_t r0 = tile / a.cblocks * a.loop, j0 = tile % a.cblocks * a.span;
    const int64_t r1 = min(r0 + a.loop, a.nq), j1 = min(j0 + a.span, a.nk);
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, threads = a.waves * 64;
    for (int e = threadIdx.x; e <= 2 * a.reach; e += threads) lut[e] = (uint8_t)bucket_of(a, e);
    for (int e = threadIdx.x; e < a.waves * table; e += threads) val[e] = 0.f;
    if (threadIdx.x < 8) touched[threadIdx.x] = 0;
    __syncthreads();
    const int c0 = cb * 64 * V + lane * V;
    const bool live = c0 < a.heads;                    // (V = 2 only where the channels are even)
    float* acc = val + (size_t)wave * table + lane;
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.f;
    int cur = -1;
    auto flush = [&]() {
        if (cur < 0) return;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            atomicAdd(acc + (cur * V + i) * 64, sum[i]);
            sum[i] = 0.f;
        }
        if (lane == 0) atomicOr(touched + cur / 32, 1u << (cur & 31));
    };
    auto turn_to = [&](int t) {
        if (t == cur) return;
        flush();
        cur = t;
    };
    const int per_row = (int)((j1 - j0 + kAhead - 1) / kAhead), steps = (int)(r1 - r0) * per_row;
    for (int g = wave; g < steps; g += a.waves) {
        const int64_t r = r0 + g / per_row, j = j0 + g % per_row * kAhead;
        const T* from = static_cast<const T*>(a.out.data) + r * a.out.row + (live ? c0 : 0);
        Vec<T, V> v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u].load(from + min(j + u, j1 - 1) * a.heads);
        const int64_t mine = min(j + (lane & (kAhead - 1)), j1 - 1);
        int t = lut[distance_index(a.pos_k[mine], a.pos_q[r], a.reach)];
        if constexpr (SEG) t = a.seg_k[mine] == a.seg_q[r] ? t : a.buckets - 1;
        const int first = __builtin_amdgcn_readfirstlane(t);
        if (j + kAhead <= j1 && __ballot(t != first) == 0) {       // one bucket for all of them: a tree
            turn_to(first);
#pragma unroll
            for (int i = 0; i < V; ++i) {
#pragma unroll
                for (int level = 0; level < 4; ++level)
#pragma unroll
                    for (int u = 0; u < 8 >> level; ++u) v[u].f[i] += v[u + (8 >> level)].f[i];
                sum[i] += v[0].f[i];
            }
        } else {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (j + u < j1) {
                    turn_to(__builtin_amdgcn_readlane(t, u));
#pragma unroll
                    for (int i = 0; i < V; ++i) sum[i] += v[u].f[i];
                }
            }
        }
    }
    flush();
    __syncthreads();
    const int64_t slot = tile * a.hblocks + cb;
    float* part = a.part + slot * table;
    for (int e = threadIdx.x; e < table; e += threads) {
        const int t = e / (64 * V);
        if (!(touched[t / 32] >> (t & 31) & 1)) continue;
        float s = 0.f;
        for (int w = 0; w < a.waves; ++w) s += val[(size_t)w * table + e];
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
        while (left) {
            const int k = __ffsll((unsigned long long)left) - 1;
            left &= left - 1;
            const float* part = a.part + ((first + 16 * k) * a.hblocks + cb) * table + t * 64 * V + lane;
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += part[64 * i];
        }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) sums[wave][64 * i + lane] = sum[i];
    __syncthreads();
    for (int e = threadIdx.x; e < 64 * V; e += 1024) {
        double s = 0;
        for (int w = 0; w < 16; ++w) s += sums[w][e];
        const int c = cb * 64 * V + (e % 64) * V + e / 64;
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

size_t lut_bytes(int reach) { return ((size_t)2 * reach + 1 + 15) & ~size_t(15); }

template <typename K>
hipError_t with_lds(K kernel, size_t lds) {
    return lds <= 65536 ? hipSuccess : hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
}

}  // namespace

int64_t relative_bias_plan(RelativeArgs& a) {
    a.tx = pow2_from(up(a.nk, 8), 256);
    const int rows = 256 / a.tx;
    const size_t entries = 2 * (size_t)a.reach + 2, per_head = (entries + entries / 8 + 1) * 4;
    a.hb = pow2_from(a.heads, 8);
    while (a.hb > 1 && a.hb * per_head > 40960) a.hb /= 2;
    a.cblocks = (int)up(a.nk, 8 * a.tx);
    auto groups = [&]() { return a.batch * up(a.heads, a.hb) * a.cblocks * up(a.nq, rows); };
    while (a.hb > 1 && groups() < 512) a.hb /= 2;
    a.loop = std::min<int64_t>(16, std::max<int64_t>(1, groups() / 2048));
    a.hblocks = (int)up(a.heads, a.hb);
    a.rblocks = up(a.nq, rows * a.loop);
    return a.batch * a.hblocks * a.cblocks * a.rblocks;
}

hipError_t launch_relative_bias(int dtype, RelativeArgs a, hipStream_t s) {
    const int64_t groups = relative_bias_plan(a);
    a.wide = strides_wide(a.base, a.batch, a.heads, a.nq) && strides_wide(a.out, a.batch, a.heads, a.nq);
    const size_t entries = 2 * (size_t)a.reach + 2, lds = (entries + entries / 8 + 1) * 4 * a.hb;
    const dim3 grid((unsigned)groups), block(256);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, grid, block, lds, s, a);
        return hipGetLastError();
    };
    const bool seg = a.seg_q, base = a.base.data;
    if (dtype == 1) return seg ? base ? go(k_relative_bias<bf16_t, true, true>) : go(k_relative_bias<bf16_t, true, false>)
                               : base ? go(k_relative_bias<bf16_t, false, true>) : go(k_relative_bias<bf16_t, false, false>);
    return seg ? base ? go(k_relative_bias<float, true, true>) : go(k_relative_bias<float, true, false>)
               : base ? go(k_relative_bias<float, false, true>) : go(k_relative_bias<float, false, false>);
}

// Work-groups, and in a the split of the rows and the waves of each: as many as 128 KB of columns allow.
int64_t relative_bias_backward_plan(RelativeArgs& a) {
    a.tx = pow2_from(up(a.nk, 8), 64);
    a.waves = std::min(4, std::max(1, 131072 / (a.buckets * 256)));
    const int64_t heads = a.batch * a.heads, rows = a.waves * (64 / a.tx);
    a.splits = (int)std::max<int64_t>(1, std::min(up(1024, std::max<int64_t>(1, heads)), up(a.nq, 4 * rows)));
    return heads * a.splits;
}
size_t relative_bias_part_floats(RelativeArgs a) {
    relative_bias_backward_plan(a);
    const int64_t slots = a.batch * a.splits;
    return slots <= 1 ? 0 : (size_t)slots * a.heads * a.buckets;
}

hipError_t launch_relative_bias_backward(int dtype, RelativeArgs a, hipStream_t s) {
    const int64_t groups = relative_bias_backward_plan(a), n = (int64_t)a.heads * a.buckets;
    if (a.batch == 0 || a.nq == 0 || a.nk == 0) {
        hipLaunchKernelGGL(k_relative_zero, dim3((unsigned)up(n, 256)), dim3(256), 0, s, a.dtable, n);
        return hipGetLastError();
    }
    a.wide = strides_wide(a.out, a.batch, a.heads, a.nq);
    const size_t lds = (size_t)a.waves * a.buckets * 256 + lut_bytes(a.reach);
    const dim3 grid((unsigned)groups), block(a.waves * 64);
    auto go = [&](auto kernel) {
        if (hipError_t e = with_lds(kernel, lds); e != hipSuccess) return e;
        hipLaunchKernelGGL(kernel, grid, block, lds, s, a);
        return hipGetLastError();
    };
    const hipError_t e = dtype == 1 ? a.seg_q ? go(k_relative_bias_backward<bf16_t, true>) : go(k_relative_bias_backward<bf16_t, false>)
                                    : a.seg_q ? go(k_relative_bias_backward<float, true>) : go(k_relative_bias_backward<float, false>);
    if (e != hipSuccess || a.batch * a.splits == 1) return e;
    hipLaunchKernelGGL(k_relative_join, dim3((unsigned)up(n, 64)), dim3(256), 0, s, a, a.batch * a.splits);
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
    a.loop = std::min<int64_t>(64, std::max<int64_t>(1, groups / 1024));
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

// Tiles of about 1 / 512 of the pairs each.
int64_t relative_pair_backward_plan(RelativeArgs& a, int vector) {
    a.hblocks = (int)up(a.heads, 64 * vector);
    a.waves = std::min(4, std::max(1, 139264 / (a.buckets * 256 * vector)));
    const double pairs = (double)a.nq * a.nk / 512;
    a.span = std::min<int64_t>(a.nk, std::max<int64_t>(64, up((int64_t)std::sqrt(pairs), 16) * 16));
    a.loop = std::max<int64_t>(1, (int64_t)std::ceil(pairs / a.span));
    if (a.loop > a.nq) {
        a.loop = a.nq;
        a.span = up((int64_t)std::ceil(pairs / a.nq), 16) * 16;
    }
    a.cblocks = (int)up(a.nk, a.span);
    a.rblocks = up(a.nq, a.loop);
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
    const size_t lds = (size_t)a.waves * a.buckets * 256 * v + 32 + lut_bytes(a.reach);
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
