// Attention of queries over keys of another length, forward: one pass over
// the keys with a running maximum M, sum L and unnormalised output,
//
//     x_ij = scale q_i . k_j + bias_ij,   out_i = sum_j exp(x_ij - M_i) v_j / L_i
//
// Scores are computed transposed, S^T = K Q^T, so that a lane holds one query
// and KC / 2 consecutive keys of each chunk of KC: maximum and sum are its own
// registers' and its partner's (lane ^ 32), its bias is contiguous, and the
// weights feed O^T += V^T P^T from the registers they are in.
//
// What bounds it, by the counters, as shares of a busy compute unit's cycles in
// products and in vector instructions (which hardly overlap on a SIMD).  Large
// calls by the issue of both in turn: at d = 128 without a bias 44% and 51% (2 entries
// x 16 heads, 4096 queries x 6000 keys, bf16: 438 to 560 us by the clock that a
// card holds, 920 to 720 TFLOP/s), at d = 32 with a bias 11% and 67% (384 x 4
// heads of 384 x 384: 98 us, 2.3e12 scores/s).  The 32-column form by waiting:
// 16 heads of 24, 1300 x 1300, 5% and 39%, its two or three waves a SIMD
// without anything to issue for half of their time (26 us); fp32, 500 x 777,
// 29% and 17% with one wave a SIMD on half the compute units (16 us).  Few queries
// over many keys by memory (8 x 16000 keys of 4 heads of 64, one query: 23 us, 5.7 TB/s).
#include "crossattn.h"

namespace trimul {
namespace {

// Waves per SIMD that the registers are limited for.
template <typename T, int DP, int WK>
constexpr int forward_waves() {
    return DP == 32 ? (WK == 1 || sizeof(T) == 2 ? 4 : 3) : DP == 64 ? (WK == 1 ? 3 : 2) : (sizeof(T) == 4 && WK == 4 ? 1 : 2);
}

// WK = 1: a wave takes 32 columns and every chunk, the chunks staged by all
// four waves (double-buffered).  WK = 4: 32 columns, wave w takes chunks w,
// w + 4, ..., stages them for itself, and the four results are merged at the end.
// SOLO (WK = 4): each wave has a key head of its own, with 32 columns at most.
// Chunks are KC = 64 keys in bf16 (32, with room for a third wave on a SIMD, was
// slower at d = 128), 32 in fp32 and where each wave has tiles of its own.
template <typename T, int DP, int KC, int WK, bool SOLO, bool BIAS>
__global__ __launch_bounds__(256, (forward_waves<T, DP, WK>())) void k_cross_forward(const CrossArgs a, int ctiles) {
    using TL = Tile<T, DP, KC>;
    constexpr int NT = 256 / WK, NB = KC / 32, ND = DP / 32, NS = DP / 16;
    __shared__ __align__(16) char mem[(WK == 1 ? 2 : 4) * 2 * TL::kBytes];
    __shared__ float red[WK == 1 || SOLO ? 1 : 2][WK == 1 || SOLO ? 1 : 4][32];
    const int lane = threadIdx.x & 63, ql = lane & 31, hi = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = WK == 1 ? threadIdx.x : lane;

    uint32_t blk = xcd_block();
    if (SOLO) {
        blk = blk * 4 + w;
        if (blk >= (uint32_t)(a.batch * a.kv_heads)) return;             // (no barrier follows in this form)
    }
    const int split = (int)(blk % (uint32_t)a.splits);
    blk /= (uint32_t)a.splits;
    const int ct = (int)(blk % (uint32_t)ctiles);
    blk /= (uint32_t)ctiles;
    const int hk = (int)(blk % (uint32_t)a.kv_heads);
    const int64_t b = blk / (uint32_t)a.kv_heads;
    const int ncols = a.nq * a.group;
    const int cw = ct * (128 / WK) + (WK == 1 ? 32 * w : 0);      // the wave's first column
    const bool wave_live = cw < ncols;
    const bool valid = cw + ql < ncols;
    const int col = min(cw + ql, ncols - 1);
    const int qi = col / a.group, h = hk * a.group + (col - qi * a.group);

    // (before the first chunk: behind it, 4% longer for 384 x 4 heads of 384 x 384, and 7% for 300 x 500 in fp32)
    Frag<T> qf[NS];
    {
        const T* row = (const T*)a.q.data + b * a.q.batch + (int64_t)qi * a.q.token + h * a.q.head;
#pragma unroll
        for (int s = 0; s < NS; ++s) load_row(row, s, hi, a.d, qf[s]);
    }
    const T* kb = (const T*)a.k.data + b * a.k.batch + hk / a.key_div * a.k.head;
    const T* vb = (const T*)a.v.data + b * a.v.batch + hk / a.key_div * a.v.head;
    const uint8_t* mask = a.mask ? a.mask + b * a.mask_batch : nullptr;
    const int ks = split * a.split_keys, ke = min(a.nk, ks + a.split_keys);
    const int nchunks = (ke - ks + KC - 1) / KC;

    // without a bias x stays in units of q . k and the scale is part of the exponential's factor
    const float coef = BIAS ? kLog2e : a.scale * kLog2e;
    f32x16_t o[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    float M = -INFINITY, L = 0.f;

    TL tl;
    tl.init(lane);
    Part<T, DP, KC, NT> kp, vp;
    KeyByte kbyte;
    BiasRow<T, KC> bp;
    kp.init(a.k.token, a.d, t);
    vp.init(a.v.token, a.d, t);
    auto load = [&](int c) {
        const int k0 = ks + c * KC;
        kp.load(kb, a.k.token, k0, a.nk, a.d);
        vp.load(vb, a.v.token, k0, a.nk, a.d);
        kbyte.load(mask, k0, a.nk, lane);
    };
    constexpr int STEP = SOLO ? 1 : WK;
    const int c0 = WK == 1 || SOLO ? 0 : w;
    load(c0);
    if (BIAS) {
        bp.init(a, b, hk, min(cw, ncols - 1), min(cw + 31, ncols - 1), qi, h, hi);
        bp.load(ks + c0 * KC, a.nk);
    }
    for (int c = c0; c < nchunks; c += STEP) {
        char* kt = mem + (WK == 1 ? (c & 1) : w) * 2 * TL::kBytes;
        char* vt = kt + TL::kBytes;
        const int k0 = ks + c * KC;
        uint64_t bits = kbyte.bits(mask, k0, ke, lane);
        if (KC == 32) bits &= 0xffffffffull;
        const bool some = bits != (KC == 64 ? ~0ull : 0xffffffffull);
        if (WK > 1) wave_sync();
        kp.stage(kt, t, some, bits);
        vp.stage(vt, t, some, bits);
        load(c + STEP);
        if (WK == 1) __syncthreads();
        else wave_sync();
        if (bits != 0 && wave_live) {
            f32x16_t s[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = 0.f;
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    Frag<T> f;
                    tl.rows(kt, n, i, f);
                    s[n] = mma(f, qf[i], s[n]);
                }
            }
            if (BIAS) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float4 bv = bp.get(n, g);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            s[n][4 * g + e] = __builtin_fmaf(s[n][4 * g + e], a.scale, f4_get(bv, e));
                    }
                bp.load(k0 + STEP * KC, a.nk);
            }
            if (some) {
                const uint32_t mine = (uint32_t)(bits >> ((KC / 2) * hi));
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[n][r] = present_or_inf(s[n][r], mine, 16 * n + r);
            }
            float cm = -INFINITY;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; r += 2) cm = fmaxf(fmaxf(cm, s[n][r]), s[n][r + 1]);
            cm = fmaxf(cm, xor32(cm));
            const float Mn = fmaxf(M, cm);
            const float Ms = Mn == -INFINITY ? 0.f : Mn;      // no key yet: every x is -inf and every weight 0
            const float alpha = __builtin_amdgcn_exp2f((M - Ms) * coef);
            L *= alpha;
            if (__any(alpha != 1.f))                          // (for a wave deep in the keys the maxima stand most of the time)
#pragma unroll
            for (int i = 0; i < ND; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
            M = Mn;
            float nsh = -Ms * coef;
            if (__any(!(fabsf(nsh) <= kFmaMax))) {            // take the difference first
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[n][r] -= Ms;
                nsh = 0.f;
            }
            float ps = 0.f;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], coef, nsh));
                    ps += s[n][r];
                }
            L += ps;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) {
                    Frag<T> pf;      // (bf16: an error of the size of out's own rounding; a second, low part would be half as many products again)
                    take8(s[n], tt, pf);
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        Frag<T> vf;
                        tl.cols(vt, n, tt, i, vf);
                        o[i] = mma(vf, pf, o[i]);
                    }
                }
        } else if (BIAS) {
            bp.load(k0 + STEP * KC, a.nk);
        }
    }

    float Lt = L + xor32(L);
    constexpr bool MERGE = WK > 1 && !SOLO;
    constexpr int groups = MERGE ? ND : ND * 4;   // groups of four channels that this lane writes, from g0 on
    int g0 = 0;
    if constexpr (MERGE) {                  // each wave ends up with a quarter of the channels
        if (!hi) {
            red[0][w][ql] = M;
            red[1][w][ql] = Lt;
        }
        __syncthreads();                    // also: every wave is done with its tiles
        const float Mn = fmaxf(fmaxf(red[0][0][ql], red[0][1][ql]), fmaxf(red[0][2][ql], red[0][3][ql]));
        const float Ms = Mn == -INFINITY ? 0.f : Mn;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += red[1][i][ql] * __builtin_amdgcn_exp2f((red[0][i][ql] - Ms) * coef);
        const float f = __builtin_amdgcn_exp2f((M - Ms) * coef);
#pragma unroll
        for (int i = 0; i < ND; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[i][r] *= f;
        add_waves<ND>(o, reinterpret_cast<float*>(mem), w, lane);
        M = Mn;
        Lt = sum;
        g0 = w * ND;
    }
    if (!valid) return;
    const int64_t row = (b * a.heads + h) * a.nq + qi;
    if (a.splits > 1) {
        const int64_t rows = a.batch * a.heads * a.nq, at = (int64_t)split * rows + row;
        store_row<ND>(a.part + at * a.d, o, groups, g0, hi, a.d, 1.f);
        if (!hi && (!MERGE || w == 0)) {
            float* pm = a.part + (int64_t)a.splits * rows * a.d;
            pm[at] = M;
            pm[(int64_t)a.splits * rows + at] = Lt;
        }
        return;
    }
    const float inv = Lt == 0.f ? 0.f : 1.f / Lt;
    store_row<ND>((T*)a.out.data + b * a.out.batch + (int64_t)qi * a.out.token + h * a.out.head, o, groups, g0, hi, a.d, inv);
    if constexpr (sizeof(T) == 2)
        if (a.stats) store_rest<ND>((bf16_t*)a.rest + row * a.d, o, groups, g0, hi, a.d, inv);
    if (a.stats && !hi && (!MERGE || w == 0)) {
        a.stats[row] = BIAS ? M : M * a.scale;
        a.stats[a.batch * a.heads * a.nq + row] = Lt;
    }
}

// The splits of one (entry, head, query) joined: out = sum_s exp(M_s - M) O_s / sum_s exp(M_s - M) L_s.
// A wave to each, a lane to each split and then to each channel; a launch's time for few rows (128 rows: 4 us).
template <typename T>
__global__ __launch_bounds__(64) void k_cross_join(const CrossArgs a) {
    __shared__ float wt[kCrossMaxSplits];
    const int64_t rows = a.batch * a.heads * a.nq, row = blockIdx.x;
    const int lane = threadIdx.x;
    const float coef = a.bias.data ? kLog2e : a.scale * kLog2e;
    const float* pm = a.part + (int64_t)a.splits * rows * a.d;
    const float m = lane < a.splits ? pm[(int64_t)lane * rows + row] : -INFINITY;
    float l = lane < a.splits ? pm[((int64_t)a.splits + lane) * rows + row] : 0.f;
    float M = m;
#pragma unroll
    for (int i = 32; i; i >>= 1) M = fmaxf(M, __shfl_xor(M, i));
    const float Ms = M == -INFINITY ? 0.f : M;
    const float f = __builtin_amdgcn_exp2f((m - Ms) * coef);
    wt[lane] = f;
    l *= f;
#pragma unroll
    for (int i = 32; i; i >>= 1) l += __shfl_xor(l, i);
    __syncthreads();
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const int qi = (int)(row % a.nq);
    const int64_t bh = row / a.nq, b = bh / a.heads;
    const int h = (int)(bh - b * a.heads);
    T* po = (T*)a.out.data + b * a.out.batch + (int64_t)qi * a.out.token + h * a.out.head;
    for (int c = lane; c < a.d; c += 64) {
        float x = 0.f;
        for (int s = 0; s < a.splits; ++s) x += wt[s] * a.part[((int64_t)s * rows + row) * a.d + c];
        Store<T>::st(po + c, x * inv);
        if constexpr (sizeof(T) == 2)
            if (a.stats) ((bf16_t*)a.rest)[row * a.d + c] = f2bf(rounded_off(x * inv));
    }
    if (a.stats && lane == 0) {
        a.stats[row] = a.bias.data ? M : M * a.scale;
        a.stats[rows + row] = l;
    }
}

template <typename T, int DP, bool BIAS>
hipError_t forward(const CrossArgs& a, const CrossPlan& p, hipStream_t s) {
    constexpr int KC = sizeof(T) == 2 ? 64 : 32;
    const int ctiles = (a.nq * a.group + p.cols - 1) / p.cols;
    const dim3 grid((unsigned)(a.batch * a.kv_heads * ctiles * p.splits));
    if (p.solo)
        hipLaunchKernelGGL((k_cross_forward<T, DP, 32, 4, true, BIAS>), dim3((grid.x + 3) / 4), dim3(256), 0, s, a, ctiles);
    else if (p.cols == 128)
        hipLaunchKernelGGL((k_cross_forward<T, DP, KC, 1, false, BIAS>), grid, dim3(256), 0, s, a, ctiles);
    else
        hipLaunchKernelGGL((k_cross_forward<T, DP, 32, 4, false, BIAS>), grid, dim3(256), 0, s, a, ctiles);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    hipLaunchKernelGGL((k_cross_join<T>), dim3((unsigned)(a.batch * a.heads * a.nq)), dim3(64), 0, s, a);
    return hipGetLastError();
}

template <typename T, int DP>
hipError_t forward(const CrossArgs& a, const CrossPlan& p, hipStream_t s) {
    return a.bias.data ? forward<T, DP, true>(a, p, s) : forward<T, DP, false>(a, p, s);
}

template <typename T>
hipError_t forward(const CrossArgs& a, const CrossPlan& p, hipStream_t s) {
    return a.d <= 32 ? forward<T, 32>(a, p, s) : a.d <= 64 ? forward<T, 64>(a, p, s) : forward<T, 128>(a, p, s);
}

}  // namespace

// A wave to each key head where all have 32 columns at most and there are four
// waves for each compute unit.
// 128 columns to a work-group where that makes one for each compute unit; else
// 32, its waves on different keys.  Where even that leaves compute units
// without one, the keys are split, for two on each, as long as a split
// keeps 512 keys (four chunks a wave): the join is a launch of 4 us, 13 for 20800
// rows of d = 24.  (fp32, 2 entries x 4 heads, 500 x 777: 16.4 us whole, 14.9 + 4.3 us in three splits.)
CrossPlan cross_plan(int64_t batch, int kv_heads, int64_t cols, int64_t nk) {
    CrossPlan p{cross_few(batch * kv_heads, cols) ? 32 : 128, 1, (int)((nk + 63) / 64 * 64), cross_solo(batch * kv_heads, cols)};
    if (p.solo) p.cols = 32;
    const int64_t groups = batch * kv_heads * ((cols + p.cols - 1) / p.cols);
    if (groups > 0 && groups < 256) {
        int64_t n = (512 + groups - 1) / groups;
        if (n > nk / 512) n = nk / 512;
        if (n > kCrossMaxSplits) n = kCrossMaxSplits;
        if (n > 1) {
            p.split_keys = (int)(((nk + n - 1) / n + 63) / 64 * 64);
            p.splits = (int)((nk + p.split_keys - 1) / p.split_keys);
        }
    }
    return p;
}

size_t cross_part_floats(const CrossPlan& p, int64_t batch, int64_t nq, int heads, int d) {
    return p.splits > 1 ? (size_t)p.splits * (size_t)batch * (size_t)nq * (size_t)heads * (size_t)(d + 2) : 0;
}

hipError_t launch_cross_forward(int dtype, const CrossArgs& args, const CrossPlan& p, hipStream_t s) {
    CrossArgs a = args;
    a.splits = p.splits;
    a.split_keys = p.split_keys;
    return dtype == 1 ? forward<bf16_t>(a, p, s) : forward<float>(a, p, s);
}

}  // namespace trimul
