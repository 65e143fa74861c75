// Residual addition with dropout, and its backward, for [rows][cols][channels]
// tensors with a mask that is computed where it is needed.
//
// One Philox call (ten rounds, 20 32 x 32 -> 64 bit products at a quarter of
// the rate) serves four elements; where a mask is shared a thread computes its
// own once and walks the axis that shares it.  Shared: bound by memory, x, res and out
// once, vector instructions 16% of a busy compute unit's cycles (2048 x 2048 x 128,
// fp32 + bf16 -> bf16, columns: 807 us, 5.3 TB/s).  Each element its own: the
// generator's 20 operations an element keep the vector units busy for 91% of the cycles, and at
// 4 bytes an element memory is as near its rate (500 x 700 x 128 bf16, backward: 32 us, 5.6 TB/s).
// Small: a launch (64 x 64 x 128 fp32: 3.5 us).
#include "common.h"
#include "kernels.h"
#include "vec.h"

namespace trimul {
namespace {

struct Words { uint32_t w[4]; };

// Philox-4x32-10: counter (e4, offset), key seed.
__device__ __forceinline__ Words philox(uint64_t e4, uint64_t offset, uint64_t seed) {
    uint32_t a = (uint32_t)e4, b = (uint32_t)(e4 >> 32), c = (uint32_t)offset, d = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = (uint64_t)a * 0xD2511F53u, p1 = (uint64_t)c * 0xCD9E8D57u;
        a = (uint32_t)(p1 >> 32) ^ b ^ k0;
        b = (uint32_t)p1;
        c = (uint32_t)(p0 >> 32) ^ d ^ k1;
        d = (uint32_t)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Words{{a, b, c, d}};
}

// Bit i: element e + i is kept (e a multiple of 4 for V > 1).
template <int V>
__device__ __forceinline__ uint32_t kept(uint64_t e, const DropoutArgs& a) {
    if constexpr (V == 1) {
        const Words w = philox(e >> 2, a.offset, a.seed);
        const uint32_t i = (uint32_t)e & 3;
        return (i == 0 ? w.w[0] : i == 1 ? w.w[1] : i == 2 ? w.w[2] : w.w[3]) >= a.threshold && a.any ? 1u : 0u;
    } else {
        uint32_t m = 0;     // (a.any asked of m at the end instead: bits are built that nothing needs, 32.3 us for 30.0)
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const Words w = philox((e >> 2) + i, a.offset, a.seed);
#pragma unroll
            for (int j = 0; j < 4; ++j) m |= (w.w[j] >= a.threshold && a.any ? 1u : 0u) << (4 * i + j);
        }
        return m;
    }
}

// TI: the dropped input, TR: the residual (null: 0), TO: the output.
template <typename TI, typename TR, typename TO, int V>
__device__ __forceinline__ void element(const Vec<TI, V>& x, const Vec<TR, V>& r, uint32_t m, float scale, TO* out) {
    Vec<TO, V> o;
#pragma unroll
    for (int i = 0; i < V; ++i) o.f[i] = (m >> i) & 1 ? __builtin_fmaf(x.f[i], scale, r.f[i]) : r.f[i];
    o.store(out);
}

// A work-group of 256 threads takes, of a.loop consecutive rows,
//   EACH, ROWS: 256 vectors (of the flattened row; the mask of ROWS once for all rows),
//   COLUMNS:    one channel vector a thread, every a.lanes-th column of a.span columns (the mask once per row).
template <typename TI, typename TO, int V, int SHARE, bool RES>
__global__ __launch_bounds__(256) void k_pair_dropout(const DropoutArgs a, const TI* x, const TO* res, TO* out) {
    const int64_t by = blockIdx.x / a.blocks;
    const int bx = (int)(blockIdx.x - by * a.blocks);
    const int64_t r0 = by * a.loop, r1 = min(r0 + a.loop, a.rows);
    if constexpr (SHARE == 2) {
        const int cv = (int)(a.channels / V);                       // channel vectors of a pair
        const int cblocks = (cv + 255) / 256, tc = min(cv, 256);
        const int jb = bx / cblocks, cb = bx - jb * cblocks;
        const int lane = threadIdx.x / tc, c = cb * 256 + (int)threadIdx.x - lane * tc;
        if (lane >= a.lanes || c >= cv) return;
        const int64_t j0 = (int64_t)jb * a.span, j1 = min(j0 + a.span, a.cols);
        for (int64_t i = r0; i < r1; ++i) {
            const uint32_t m = kept<V>((uint64_t)((a.row0 + i) * a.n_cols * a.channels + (int64_t)c * V), a);
            const TI* px = x + i * a.ld_in + c * V;
            const TO* pr = RES ? res + i * a.ld_res + c * V : nullptr;
            TO* po = out + i * a.ld_res_out + c * V;
            int64_t j = j0 + lane;
            for (; j + 3 * a.lanes < j1; j += 4 * a.lanes) {       // four vectors in flight
                Vec<TI, V> vx[4];
                Vec<TO, V> vr[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int64_t at = (j + u * a.lanes) * a.channels;
                    vx[u].load(px + at);
                    if constexpr (RES) vr[u].load(pr + at);
                    else
#pragma unroll
                        for (int q = 0; q < V; ++q) vr[u].f[q] = 0.f;
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) element(vx[u], vr[u], m, a.scale, po + (j + u * a.lanes) * a.channels);
            }
            for (; j < j1; j += a.lanes) {
                Vec<TI, V> vx;
                Vec<TO, V> vr;
                vx.load(px + j * a.channels);
#pragma unroll
                for (int q = 0; q < V; ++q) vr.f[q] = 0.f;
                if constexpr (RES) vr.load(pr + j * a.channels);
                element(vx, vr, m, a.scale, po + j * a.channels);
            }
        }
    } else {
        const int64_t at = ((int64_t)bx * 256 + threadIdx.x) * V;   // in the flattened row
        if (at >= a.cols * a.channels) return;
        const uint64_t e0 = (uint64_t)(a.col0 * a.channels + at);
        uint32_t m = SHARE == 1 ? kept<V>(e0, a) : 0;
        auto load = [&](int64_t i, Vec<TI, V>& vx, Vec<TO, V>& vr) {
            vx.load(x + i * a.ld_in + at);
            if constexpr (RES) vr.load(res + i * a.ld_res + at);
            else
#pragma unroll
                for (int q = 0; q < V; ++q) vr.f[q] = 0.f;
        };
        int64_t i = r0;
        for (; i + 3 < r1; i += 4) {
            Vec<TI, V> vx[4];
            Vec<TO, V> vr[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) load(i + u, vx[u], vr[u]);
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (SHARE == 0) m = kept<V>((uint64_t)((a.row0 + i + u) * a.n_cols * a.channels) + e0, a);
                element(vx[u], vr[u], m, a.scale, out + (i + u) * a.ld_res_out + at);
            }
        }
        for (; i < r1; ++i) {
            Vec<TI, V> vx;
            Vec<TO, V> vr;
            load(i, vx, vr);
            if (SHARE == 0) m = kept<V>((uint64_t)((a.row0 + i) * a.n_cols * a.channels) + e0, a);
            element(vx, vr, m, a.scale, out + i * a.ld_res_out + at);
        }
    }
}

// The largest vector that the channels, the row strides and the pointers allow.
int vector_of(const DropoutArgs& a, const void* x, const void* res, const void* out) {
    const int64_t bits = a.channels | a.ld_in | a.ld_res_out | (res ? a.ld_res : 0);
    const uintptr_t ptr = reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(res) | reinterpret_cast<uintptr_t>(out);
    if (ptr & 15) return 1;
    return bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 1;
}

// About 2048 work-groups (eight a compute unit) before a work-group takes more rows (up to 16).
int64_t rows_per_group(int64_t rows, int64_t blocks) {
    const int64_t n = rows * blocks / 2048;
    return n < 1 ? 1 : n > 16 ? 16 : n;
}

template <typename TI, typename TO, int V, bool RES>
hipError_t launch(DropoutArgs a, int share, const void* x, const void* res, void* out, hipStream_t s) {
    if (share == 2) {
        const int64_t cv = a.channels / V, tc = cv < 256 ? cv : 256, cblocks = (cv + 255) / 256;
        a.lanes = (int)(256 / tc);
        a.span = 8 * a.lanes;                                       // eight vectors a thread
        a.blocks = (int)((a.cols + a.span - 1) / a.span * cblocks);
        a.loop = 1;
    } else {
        a.blocks = (int)((a.cols * a.channels / V + 255) / 256);
        a.loop = rows_per_group(a.rows, a.blocks);
    }
    // more rows each where the grid would outgrow 2^24 work-groups (blocks stays below 2^23: a row is below 2^31)
    const int64_t most = (int64_t(1) << 24) / a.blocks - 1;
    if ((a.rows + a.loop - 1) / a.loop > most) a.loop = (a.rows + most - 1) / most;
    const int64_t groups = (a.rows + a.loop - 1) / a.loop * a.blocks;
    const dim3 grid((unsigned)groups), block(256);
    if (share == 0) hipLaunchKernelGGL((k_pair_dropout<TI, TO, V, 0, RES>), grid, block, 0, s, a, (const TI*)x, (const TO*)res, (TO*)out);
    else if (share == 1) hipLaunchKernelGGL((k_pair_dropout<TI, TO, V, 1, RES>), grid, block, 0, s, a, (const TI*)x, (const TO*)res, (TO*)out);
    else hipLaunchKernelGGL((k_pair_dropout<TI, TO, V, 2, RES>), grid, block, 0, s, a, (const TI*)x, (const TO*)res, (TO*)out);
    return hipGetLastError();
}

template <typename TI, typename TO>
hipError_t launch(const DropoutArgs& a, int share, const void* x, const void* res, void* out, hipStream_t s) {
    const int v = vector_of(a, x, res, out);
    if (res) return v == 8 ? launch<TI, TO, 8, true>(a, share, x, res, out, s) : v == 4 ? launch<TI, TO, 4, true>(a, share, x, res, out, s) : launch<TI, TO, 1, true>(a, share, x, res, out, s);
    return v == 8 ? launch<TI, TO, 8, false>(a, share, x, res, out, s) : v == 4 ? launch<TI, TO, 4, false>(a, share, x, res, out, s) : launch<TI, TO, 1, false>(a, share, x, res, out, s);
}

}  // namespace

hipError_t launch_pair_dropout(int in_dtype, int out_dtype, int share, const DropoutArgs& a, const void* x,
                               const void* res, void* out, hipStream_t s) {
    if (in_dtype == 1) return out_dtype == 1 ? launch<bf16_t, bf16_t>(a, share, x, res, out, s) : launch<bf16_t, float>(a, share, x, res, out, s);
    return out_dtype == 1 ? launch<float, bf16_t>(a, share, x, res, out, s) : launch<float, float>(a, share, x, res, out, s);
}

}  // namespace trimul
