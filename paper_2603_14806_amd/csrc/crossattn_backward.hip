// Attention of queries over keys of another length, backward.  From the
// forward's M_i and L_i the weights are P_ij = exp(x_ij - M_i) / L_i again, and
//
//     D_i = dout_i . out_i        dS_ij = P_ij (dout_i . v_j - D_i)
//     dq_i = scale sum_j dS_ij k_j        dbias = dS, summed where a bias is shared
//     dk_j = scale sum_i dS_ij q_i        dv_j = sum_i P_ij dout_i
//
// Three passes, each the owner of what it writes, so that every sum has one
// order and nothing is added atomically (the first two side by side in one
// launch where they are small): queries (dq, and D for the others),
// keys (dk, dv; a key head's loop runs over the columns of all its query
// heads) and, where a bias is given, tiles of it (whose loop runs over the
// entries and heads that share it).  Each recomputes S and dP: writing dS
// down instead would cost more than it saves (384 entries x 4 heads of 384 x 384 in
// bf16: 0.45 GB, 180 us there and back, against a pass's 100).
#include "crossattn.h"

#include <algorithm>
#include <cmath>

namespace trimul {
namespace {

// A query's statistics as the weights use them: P = exp2((x - M) log2 e + n2) = exp2(x log2 e + sh).
// A query with no key: M = 0, n2 = -inf, P = 0.  The query pass (or k_cross_rows) leaves them, and D, in the workspace
// for the other two.
struct RowStat {
    float M, n2, sh, D;
    __device__ __forceinline__ void set(float m, float l, float d) {
        M = l == 0.f ? 0.f : m;
        n2 = l == 0.f ? -INFINITY : -__builtin_amdgcn_logf(l);
        sh = __builtin_fmaf(-M, kLog2e, n2);
        D = d;
    }
    __device__ __forceinline__ bool far() const { return !(fabsf(M * kLog2e) <= kFmaMax); }
};

// x = q . k scale + bias of a lane's 16 keys of the n-th 32.
template <typename T, int KC>
__device__ __forceinline__ void add_bias(f32x16_t& s, int n, const BiasRow<T, KC>& bp, float scale) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const float4 bv = bp.get(n, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[4 * g + e] = __builtin_fmaf(s[4 * g + e], scale, f4_get(bv, e));
    }
}
// Absent keys (their bit of `mine` is 0): x = -inf.
__device__ __forceinline__ void drop_absent(f32x16_t& s, uint32_t mine) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = present_or_inf(s[r], mine, r);
}
// x - M where M is large.
__device__ __forceinline__ void take_from(f32x16_t& s, float scale, float M) {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = __builtin_fmaf(s[r], scale, -M);
}

// ------------------------------------------------------------------ queries: dq, D
//
// The forward's layout (lane: one column, registers: keys): WK = 1, 32 columns
// a wave, or WK = 4, 32 columns a work-group and its waves on different keys, or
// SOLO (WK = 4), a key head of 32 columns at most for each wave.
// A bias that no other entry or head shares gets its gradient, dS, from here (DIRECT; asked
// at each product instead, the branches there cut the others' code into pieces).
// Three products a score and channel, and the exponential.  At d = 32 with few keys not bound by their issue
// (products 14%, vector instructions 51% of a busy compute unit's cycles) but by the rows that each work-group
// waits for at its start and its bias loads (384 entries x 4 heads of 384 x 384, bias: 118 us; without the
// exponentials it took 120 of 121 us, without any loads 96).  At d = 128 products and vector instructions are
// 41% and 37% (2 entries x 16 heads, 2048 x 3000: 158 us, 480 TFLOP/s).
template <typename T, int DP, int WK>
constexpr int q_waves() {
    if (WK > 1) return sizeof(T) == 2 ? (DP == 32 ? 3 : DP == 64 ? 2 : 1) : (DP == 32 ? 2 : 1);
    return DP == 32 ? 3 : DP == 64 || sizeof(T) == 2 ? 2 : 1;
}

// LDS bytes of a work-group.
template <typename T, int DP, int KC, int WK>
constexpr int q_lds() { return (WK == 1 ? 2 : 4) * 2 * Tile<T, DP, KC>::kBytes; }

// ROWS: leaves the statistics for the passes behind it (else k_cross_rows has done so).
template <typename T, int DP, int KC, int WK, bool SOLO, bool BIAS, bool DIRECT, bool ROWS>
__device__ __forceinline__ void query_pass(const CrossArgs& a, int ctiles, uint32_t blk, char* mem) {
    using TL = Tile<T, DP, KC>;
    constexpr int NT = 256 / WK, NB = KC / 32, ND = DP / 32, NS = DP / 16;
    constexpr bool FOLD = sizeof(T) == 2 && DP <= 64;          // dP's sum starts at -D (16 registers that hold it)
    const int lane = threadIdx.x & 63, ql = lane & 31, hi = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = WK == 1 ? threadIdx.x : lane;

    if (SOLO) {
        blk = blk * 4 + w;
        if (blk >= (uint32_t)(a.batch * a.kv_heads)) return;             // (no barrier follows in this form)
    }
    const int ct = (int)(blk % (uint32_t)ctiles);
    blk /= (uint32_t)ctiles;
    const int hk = (int)(blk % (uint32_t)a.kv_heads);
    const int64_t b = blk / (uint32_t)a.kv_heads;
    const int ncols = a.nq * a.group, cw = ct * (128 / WK) + (WK == 1 ? 32 * w : 0);
    const bool wave_live = cw < ncols, valid = cw + ql < ncols;
    const int col = min(cw + ql, ncols - 1);
    const int qi = col / a.group, h = hk * a.group + (col - qi * a.group);
    const int64_t row = (b * a.heads + h) * a.nq + qi;

    constexpr bool MERGE = WK > 1 && !SOLO;
    constexpr int STEP = MERGE ? WK : 1;
    const float coef = BIAS ? kLog2e : a.scale * kLog2e;
    const T* kb = (const T*)a.k.data + b * a.k.batch + hk / a.key_div * a.k.head;
    const T* vb = (const T*)a.v.data + b * a.v.batch + hk / a.key_div * a.v.head;
    const uint8_t* mask = a.mask ? a.mask + b * a.mask_batch : nullptr;
    const int nchunks = (a.nk + KC - 1) / KC;
    T* const drow = DIRECT ? (T*)a.dbias.data + b * a.dbias.batch + h * a.dbias.head + (int64_t)qi * a.dbias.row : nullptr;

    // the first chunk is asked for before the rows' own values are waited for
    TL tl;
    tl.init(lane);
    Part<T, DP, KC, NT> kp, vp;
    KeyByte kbyte;
    BiasRow<T, KC> bp;
    kp.init(a.k.token, a.d, t);
    vp.init(a.v.token, a.d, t);
    auto load = [&](int c) {
        kp.load(kb, a.k.token, c * KC, a.nk, a.d);
        vp.load(vb, a.v.token, c * KC, a.nk, a.d);
        kbyte.load(mask, c * KC, a.nk, lane);
    };
    const int c0 = MERGE ? w : 0;
    load(c0);
    if (BIAS) {
        bp.init(a, b, hk, min(cw, ncols - 1), min(cw + 31, ncols - 1), qi, h, hi);
        bp.load(c0 * KC, a.nk);
    }

    Frag<T> qf[NS], gf[NS];
    float D = 0.f;
    {
        const T* qr = (const T*)a.q.data + b * a.q.batch + (int64_t)qi * a.q.token + h * a.q.head;
        const T* gr = (const T*)a.dout.data + b * a.dout.batch + (int64_t)qi * a.dout.token + h * a.dout.head;
        const T* orow = (const T*)a.out.data + b * a.out.batch + (int64_t)qi * a.out.token + h * a.out.head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            Frag<T> of;
            load_row(qr, s, hi, a.d, qf[s]);
            load_row(gr, s, hi, a.d, gf[s]);
            load_row(orow, s, hi, a.d, of);
            D += Frag<T>::dot(gf[s], of);
            if constexpr (sizeof(T) == 2) {
                load_row((const bf16_t*)a.rest + row * a.d, s, hi, a.d, of);
                D += Frag<T>::dot(gf[s], of);
            }
        }
        D += xor32(D);
    }
    RowStat st;
    st.set(a.stats[row], a.stats[a.batch * a.heads * a.nq + row], D);
    if (ROWS && valid && !hi && (!MERGE || w == 0)) reinterpret_cast<float4*>(a.rows)[row] = make_float4(st.M, st.n2, st.sh, D);
    const bool far = __any(st.far());
    f32x16_t acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;

    f32x16_t start;
#pragma unroll
    for (int r = 0; r < 16; ++r) start[r] = FOLD ? -D : 0.f;

    for (int c = c0; c < nchunks; c += STEP) {
        char* kt = mem + (WK == 1 ? (c & 1) : w) * 2 * TL::kBytes;
        char* vt = kt + TL::kBytes;
        uint64_t bits = kbyte.bits(mask, c * KC, a.nk, lane);
        if (KC == 32) bits &= 0xffffffffull;
        const bool some = bits != (KC == 64 ? ~0ull : 0xffffffffull);
        if (WK > 1) wave_sync();
        kp.stage(kt, t, some, bits);
        vp.stage(vt, t, some, bits);
        load(c + STEP);
        if (WK == 1) __syncthreads();
        else wave_sync();
        if (bits != 0 && wave_live) {
            const uint32_t mine = (uint32_t)(bits >> ((KC / 2) * hi));
#pragma unroll
            for (int n = 0; n < NB; ++n) {                     // 32 keys at a time: their scores are all that is live
                f32x16_t s, dp = start;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    Frag<T> f;
                    tl.rows(kt, n, i, f);
                    s = mma(f, qf[i], s);
                }
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    Frag<T> f;
                    tl.rows(vt, n, i, f);
                    dp = mma(f, gf[i], dp);
                }
                if (BIAS) {
                    add_bias<T, KC>(s, n, bp, a.scale);
                    if (n == NB - 1) bp.load((c + STEP) * KC, a.nk);
                }
                if (some) drop_absent(s, mine >> (16 * n));
                float cf = coef, sh = st.sh;
                if (far) {
                    take_from(s, BIAS ? 1.f : a.scale, st.M);
                    cf = kLog2e;
                    sh = st.n2;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], cf, sh)) * (FOLD ? dp[r] : dp[r] - D);
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) {
                    Frag<T> pf;                                // (bf16: dS is rounded for its product as dq is for its store)
                    take8(s, tt, pf);
                    if (DIRECT) {
                        const int k = c * KC + (KC / 2) * hi + 16 * n + 8 * tt;
                        if (valid) store8(drow + k, pf, a.nk - k);
                    }
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        Frag<T> kf;
                        tl.cols(kt, n, tt, i, kf);
                        acc[i] = mma(kf, pf, acc[i]);
                    }
                }
            }
        } else if (BIAS) {
            bp.load((c + STEP) * KC, a.nk);
            if (DIRECT && valid) {                      // no key here: dS is 0
                Frag<T> z;
                z.zero();
#pragma unroll
                for (int i = 0; i < KC / 16; ++i) {
                    const int k = c * KC + (KC / 2) * hi + 8 * i;
                    store8(drow + k, z, a.nk - k);
                }
            }
        }
    }
    if constexpr (MERGE) {
        __syncthreads();
        add_waves<ND>(acc, reinterpret_cast<float*>(mem), w, lane);
    }
    if (!valid) return;
    store_row<ND>((T*)a.dq.data + b * a.dq.batch + (int64_t)qi * a.dq.token + h * a.dq.head, acc, MERGE ? ND : 4 * ND,
                  MERGE ? w * ND : 0, hi, a.d, a.scale);
}

template <typename T, int DP, int KC, int WK, bool SOLO, bool BIAS, bool DIRECT>
__global__ __launch_bounds__(256, (q_waves<T, DP, WK>())) void k_cross_backward_q(const CrossArgs a, int ctiles) {
    __shared__ __align__(16) char mem[q_lds<T, DP, KC, WK>()];
    query_pass<T, DP, KC, WK, SOLO, BIAS, DIRECT, true>(a, ctiles, xcd_block(), mem);
}

// ------------------------------------------------------------------ keys: dk, dv
//
// Lane: one key (K and V as B operands in registers), registers: the queries of
// a chunk of QC (of one head after the other), whose q and dout pass through
// LDS: WK = 1, 32 keys a wave, or WK = 4, 32 keys a work-group and its waves on
// different chunks.  TWO (WK = 1): eight waves, each 32 keys taken by two of
// them, one for dv (S and P^T dout), one for dk (S, dP and dS^T Q).  S twice
// is a quarter more products, but at d = 128 the two sums and the fragments of
// K and V leave no room for a second wave on a SIMD, and a single one waits
// for each of its LDS reads and products in turn.
// The bias tile of a chunk passes through LDS too and is read transposed
// (four queries of one key at a time).
// Bound by instruction issue: four products a score and channel (TWO: five)
// and their LDS reads (products 20%, vector instructions 55%, LDS 13% of a busy compute unit's cycles: 384 entries
// x 4 heads of 384 x 384, d = 32, bias: 139 us).  TWO: 38%, 34% and 11%, its two waves a SIMD waiting for each
// other's chunk the rest (2 entries x 16 heads on 4, 2048 x 3000, d = 128: 303 to 316 us and 18 for the sums of four splits).
template <typename T, int DP, int WK, bool TWO>
constexpr int kv_waves() { return TWO ? 2 : DP == 32 ? (sizeof(T) == 2 ? 3 : 2) : DP == 64 && sizeof(T) == 2 ? 2 : 1; }

// LDS of a work-group: tiles, bias rows (four of them spread over the banks), statistics.
template <typename T, int DP, int QC, int WK, bool BIAS>
struct KvLds {
    static constexpr int kBuf = WK == 1 ? 2 : 4, kKeys = 128 / WK;
    static constexpr int kBRow = kKeys * (int)sizeof(T) + (sizeof(T) == 4 ? 16 : kKeys == 128 ? 64 : 0);
    static constexpr int kBias = kBuf * 2 * Tile<T, DP, QC>::kBytes, kStat = kBias + (BIAS ? kBuf * QC * kBRow : 0);
    static constexpr int kBytes = kStat + kBuf * 4 * QC * 4;
};

template <typename T, int DP, int QC, int WK, bool TWO, bool BIAS>
__device__ __forceinline__ void key_pass(const CrossArgs& a, int ktiles, uint32_t blk, char* mem) {
    using TL = Tile<T, DP, QC>;
    using LD = KvLds<T, DP, QC, WK, BIAS>;
    constexpr int NB = QC / 32, ND = DP / 32, NS = DP / 16;
    constexpr int NT = (TWO ? 512 : 256) / WK, KT = LD::kKeys;   // threads of a chunk, keys
    constexpr int kBRow = LD::kBRow, kBPieces = KT * (int)sizeof(T) / 16, kBN = QC * kBPieces / NT;
    char* const bmem = mem + LD::kBias;
    float(* const stat)[4][QC] = reinterpret_cast<float(*)[4][QC]>(mem + LD::kStat);   // M, n2, sh, -D of a chunk's columns
    const int lane = threadIdx.x & 63, kl = lane & 31, hi = lane >> 5;
    const int wid = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), t = WK == 1 ? threadIdx.x : lane;
    const int w = TWO ? wid & 3 : wid;
    const bool for_k = TWO && wid >= 4;                        // TWO: this wave's half

    const int kt_ = (int)(blk % (uint32_t)ktiles);
    blk /= (uint32_t)ktiles;
    const int split = (int)(blk % (uint32_t)a.splits);
    blk /= (uint32_t)a.splits;
    const int kv_heads = a.kv_heads / a.key_div, group = a.group * a.key_div;
    const int hk = (int)(blk % (uint32_t)kv_heads);
    const int64_t b = blk / (uint32_t)kv_heads;
    const int key0 = kt_ * KT, kw = WK == 1 ? 32 * w : 0, key = key0 + kw + kl;
    const bool valid = key < a.nk, wave_live = key0 + kw < a.nk;
    const int kc = min(key, a.nk - 1);
    const bool present = valid && (!a.mask || a.mask[b * a.mask_batch + kc] != 0);
    const bool all_present = __all(present);
    const int per_head = (a.nq + QC - 1) / QC, all = per_head * group;
    const int c0 = (int)((int64_t)all * split / a.splits), nchunks = (int)((int64_t)all * (split + 1) / a.splits);
    const float coef = BIAS ? kLog2e : a.scale * kLog2e;

    Frag<T> kf[NS], vf[NS];
    {
        const T* kr = (const T*)a.k.data + b * a.k.batch + (int64_t)kc * a.k.token + hk * a.k.head;
        const T* vr = (const T*)a.v.data + b * a.v.batch + (int64_t)kc * a.v.token + hk * a.v.head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            load_row(kr, s, hi, a.d, kf[s]);
            load_row(vr, s, hi, a.d, vf[s]);
            if (!present) {                                    // may hold anything
                kf[s].zero();
                vf[s].zero();
            }
        }
    }
    f32x16_t dk[TWO ? 1 : ND], dv[ND];                         // TWO: dv is the wave's one sum, dv's or dk's
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[TWO ? 0 : i][r] = dv[i][r] = 0.f;

    TL tl;
    tl.init(lane);
    Part<T, DP, QC, NT> qp, gp;
    uint4 bp[BIAS ? kBN : 1];
    uint32_t boff[BIAS ? kBN : 1];
    qp.init(a.q.token, a.d, t);
    gp.init(a.dout.token, a.d, t);
    if (BIAS)
#pragma unroll
        for (int i = 0; i < kBN; ++i) {
            const int u = t + NT * i, k = key0 + (u % kBPieces) * TL::kPer;
            boff[i] = k < a.nk ? (uint32_t)(u / kBPieces) * (uint32_t)(a.bias.row * (int)sizeof(T)) + 16 * (u % kBPieces) : 0xfffffff0u;
        }
    float4 row4 = make_float4(0.f, 0.f, 0.f, 0.f);              // the statistics of row lane % QC of the chunk
    const int first = c0 + (WK == 1 ? 0 : w);                  // this wave's first chunk
    int next_h = hk * group, next_q = 0;                       // the chunk that load() takes
    auto wrap = [&]() {
        while (next_q >= per_head * QC) {
            next_q -= per_head * QC;
            ++next_h;
        }
    };
    auto load = [&]() {
        const int left = next_h < (hk + 1) * group ? a.nq : 0;  // behind the last chunk nothing is read
        const int h = min(next_h, (hk + 1) * group - 1);
        qp.load((const T*)a.q.data + b * a.q.batch + h * a.q.head, a.q.token, next_q, left, a.d);
        gp.load((const T*)a.dout.data + b * a.dout.batch + h * a.dout.head, a.dout.token, next_q, left, a.d);
        if (BIAS) {
            const auto r = make_rsrc((const T*)a.bias.data + b * a.bias.batch + h * a.bias.head + (int64_t)next_q * a.bias.row + key0,
                                     left ? (uint32_t)((min(left - next_q, QC) - 1) * (uint32_t)a.bias.row + min(KT, (a.nk - key0 + 7) & ~7)) * (uint32_t)sizeof(T) : 0u);
#pragma unroll
            for (int i = 0; i < kBN; ++i) bp[i] = buf_load16(r, boff[i]);
        }
        const int qi = next_q + (lane & (QC - 1));
        row4 = reinterpret_cast<const float4*>(a.rows)[(b * a.heads + h) * a.nq + min(qi, a.nq - 1)];
        if (qi >= a.nq) row4.y = row4.z = -INFINITY;           // rows past the last have weight 0
        next_q += WK * QC;
        wrap();
    };
    if (c0 < nchunks) {                     // (a head has chunks then: wrap() ends)
        next_h += first / per_head;
        next_q = first % per_head * QC;
        load();
    }
    for (int c = first; c < nchunks; c += WK) {
        const int buf = WK == 1 ? c & 1 : w;
        char* qt = mem + buf * 2 * TL::kBytes;
        char* gt = qt + TL::kBytes;
        char* bt = bmem + (BIAS ? buf * QC * kBRow : 0);
        if (WK > 1) wave_sync();
        qp.stage(qt, t, false, 0);
        gp.stage(gt, t, false, 0);
        if (BIAS)
#pragma unroll
            for (int i = 0; i < kBN; ++i) {
                const int u = t + NT * i;
                *reinterpret_cast<uint4*>(bt + (u / kBPieces) * kBRow + (u % kBPieces) * 16) = bp[i];
            }
        const bool far = __any(!(fabsf(row4.x * kLog2e) <= kFmaMax));
        if ((WK > 1 || wid == 0) && lane < QC) {
            stat[buf][0][lane] = row4.x;
            stat[buf][1][lane] = row4.y;
            stat[buf][2][lane] = row4.z;
            stat[buf][3][lane] = -row4.w;
        }
        load();
        if (WK == 1) __syncthreads();
        else wave_sync();
        if (!wave_live) continue;
        const int lr = (QC / 2) * hi;                          // the lane's first tile row
        f32x16_t s[NB], dp[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[n][r] = dp[n][r] = 0.f;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                Frag<T> f;
                tl.rows(qt, n, i, f);
                s[n] = mma(f, kf[i], s[n]);
            }
            if (!TWO || for_k) {                               // dP - D: the sum starts at -D
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 d4 = *reinterpret_cast<const float4*>(&stat[buf][3][lr + 16 * n + 4 * g]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) dp[n][4 * g + e] = f4_get(d4, e);
                }
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    Frag<T> f;
                    tl.rows(gt, n, i, f);
                    dp[n] = mma(f, vf[i], dp[n]);
                }
            }
        }
        if constexpr (BIAS) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const char* p = bt + (lr + 16 * n + 4 * g) * kBRow;
                    float4 bv;
                    if constexpr (sizeof(T) == 2) {
                        const uint2 x = lds_tr4(p + ((lane >> 2) & 3) * kBRow + (kw + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2);
                        bv = bf4(x.x, x.y);
                    } else {
                        p += (kw + kl) * 4;
                        bv = make_float4(*(const float*)p, *(const float*)(p + kBRow), *(const float*)(p + 2 * kBRow),
                                         *(const float*)(p + 3 * kBRow));
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][4 * g + e] = __builtin_fmaf(s[n][4 * g + e], a.scale, f4_get(bv, e));
                }
        }
        if (!all_present) {                                    // an absent key's bias may hold anything
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = present ? s[n][r] : -INFINITY;
        }
        float cf = coef;
        const float* shifts = stat[buf][2];
        if (far) {
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4 m4 = *reinterpret_cast<const float4*>(&stat[buf][0][lr + 16 * n + 4 * g]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[n][4 * g + e] = __builtin_fmaf(s[n][4 * g + e], BIAS ? 1.f : a.scale, -f4_get(m4, e));
                }
            cf = kLog2e;
            shifts = stat[buf][1];
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 h4 = *reinterpret_cast<const float4*>(&shifts[lr + 16 * n + 4 * g]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[n][4 * g + e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][4 * g + e], cf, f4_get(h4, e)));
            }
        if (!TWO || for_k)
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    if (TWO) s[n][r] *= dp[n][r];
                    else dp[n][r] *= s[n][r];
                }
        const char* vt = TWO && for_k ? qt : gt;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                Frag<T> pf, df;                                // (bf16: P and dS rounded for their products as dv and dk for their stores)
                take8(s[n], tt, pf);
                if (!TWO) take8(dp[n], tt, df);
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    Frag<T> f;
                    tl.cols(vt, n, tt, i, f);
                    dv[i] = mma(f, pf, dv[i]);
                    if (!TWO) {
                        tl.cols(qt, n, tt, i, f);
                        dk[TWO ? 0 : i] = mma(f, df, dk[TWO ? 0 : i]);
                    }
                }
            }
    }
    if constexpr (WK > 1) {
        __syncthreads();
        add_waves<ND>(dk, reinterpret_cast<float*>(mem), w, lane);
        __syncthreads();
        add_waves<ND>(dv, reinterpret_cast<float*>(mem), w, lane);
    }
    if (!valid) return;
    constexpr int groups = WK == 1 ? 4 * ND : ND;
    const int g0 = WK == 1 ? 0 : w * ND;
    if (a.splits > 1) {                     // [split][dk, dv][entry][key head][key][d]
        const int64_t one = a.batch * kv_heads * a.nk * a.d;
        float* po = a.part + (int64_t)split * 2 * one + ((b * kv_heads + hk) * a.nk + key) * a.d;
        if (TWO) {
            store_row<ND>(for_k ? po : po + one, dv, groups, g0, hi, a.d, for_k ? a.scale : 1.f);
        } else {
            store_row<TWO ? 1 : ND>(po, dk, groups, g0, hi, a.d, a.scale);
            store_row<ND>(po + one, dv, groups, g0, hi, a.d, 1.f);
        }
        return;
    }
    T* const to_k = (T*)a.dk.data + b * a.dk.batch + (int64_t)key * a.dk.token + hk * a.dk.head;
    T* const to_v = (T*)a.dv.data + b * a.dv.batch + (int64_t)key * a.dv.token + hk * a.dv.head;
    if (TWO) {
        store_row<ND>(for_k ? to_k : to_v, dv, groups, g0, hi, a.d, for_k ? a.scale : 1.f);
    } else {
        store_row<TWO ? 1 : ND>(to_k, dk, groups, g0, hi, a.d, a.scale);
        store_row<ND>(to_v, dv, groups, g0, hi, a.d, 1.f);
    }
}

template <typename T, int DP, int QC, int WK, bool TWO, bool BIAS>
__global__ __launch_bounds__(TWO ? 512 : 256, (kv_waves<T, DP, WK, TWO>())) void k_cross_backward_kv(const CrossArgs a, int ktiles) {
    __shared__ __align__(16) char mem[KvLds<T, DP, QC, WK, BIAS>::kBytes];
    key_pass<T, DP, QC, WK, TWO, BIAS>(a, ktiles, xcd_block(), mem);
}

// ------------------------------------------------------------------ both at once
//
// Where neither pass fills the compute units they run side by side in one
// launch; what the query pass would have left for the key pass comes from a
// short launch of its own before it, 16 lanes of 8 channels to a row.
template <typename T>
__global__ __launch_bounds__(256) void k_cross_rows(const CrossArgs a) {
    const int64_t rows = a.batch * a.heads * a.nq, at = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4), row = min(at, rows - 1);
    const int64_t bh = row / a.nq, b = bh / a.heads;
    const int qi = (int)(row - bh * a.nq), h = (int)(bh - b * a.heads), l = threadIdx.x & 15;
    const T* gr = (const T*)a.dout.data + b * a.dout.batch + (int64_t)qi * a.dout.token + h * a.dout.head;
    const T* orow = (const T*)a.out.data + b * a.out.batch + (int64_t)qi * a.out.token + h * a.out.head;
    Frag<T> g, o;
    load_row(gr, 0, l, a.d, g);             // (channels 8 l ..)
    load_row(orow, 0, l, a.d, o);
    float D = Frag<T>::dot(g, o);
    if constexpr (sizeof(T) == 2) {
        load_row((const bf16_t*)a.rest + row * a.d, 0, l, a.d, o);
        D += Frag<T>::dot(g, o);
    }
#pragma unroll
    for (int i = 8; i; i >>= 1) D += __shfl_xor(D, i);
    RowStat st;
    st.set(a.stats[row], a.stats[rows + row], D);
    if (l == 0 && at < rows) reinterpret_cast<float4*>(a.rows)[row] = make_float4(st.M, st.n2, st.sh, D);
}

template <typename T, int DP, bool BIAS, bool DIRECT>
__global__ __launch_bounds__(256, (q_waves<T, DP, 4>() < kv_waves<T, DP, 4, false>() ? q_waves<T, DP, 4>() : kv_waves<T, DP, 4, false>()))
void k_cross_backward_both(const CrossArgs a, int ctiles, int ktiles, int q_blocks) {
    constexpr int kQ = q_lds<T, DP, 32, 4>(), kKv = KvLds<T, DP, 32, 4, BIAS>::kBytes;
    __shared__ __align__(16) char mem[kQ > kKv ? kQ : kKv];
    const uint32_t blk = xcd_block();
    if (blk < (uint32_t)q_blocks) query_pass<T, DP, 32, 4, false, BIAS, DIRECT, false>(a, ctiles, blk, mem);
    else key_pass<T, DP, 32, 4, false, BIAS>(a, ktiles, blk - (uint32_t)q_blocks, mem);
}

// The splits' sums of dk and dv, four channels a thread, in the order of the splits.
template <typename T>
__global__ __launch_bounds__(256) void k_cross_kv_sum(const CrossArgs a, int kv_heads) {
    const int64_t one = a.batch * kv_heads * a.nk * a.d, i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4;
    if (i >= 2 * one) return;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < a.splits; ++s) {
        const float4 y = *reinterpret_cast<const float4*>(a.part + (int64_t)s * 2 * one + i);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    const bool is_v = i >= one;
    const int64_t r = (is_v ? i - one : i) / a.d, bh = r / a.nk, b = bh / kv_heads;
    const int c = (int)(i % a.d), key = (int)(r - bh * a.nk), hk = (int)(bh - b * kv_heads);
    const CrossTensor& to = is_v ? a.dv : a.dk;
    store4((T*)to.data + b * to.batch + (int64_t)key * to.token + hk * to.head + c, x.x, x.y, x.z, x.w);
}

// ------------------------------------------------------------------ dbias
//
// A bias that several entries or heads share.  One work-group: 128 queries x KC keys of it (the query
// pass's layout), its loop over the entries and heads that share it (a split of them: the sums of the splits are added by
// k_cross_dbias_sum).  Bound by issue (products 12%, vector instructions 46%, LDS 10% of a busy compute unit's
// cycles) and the latency of its 64 keys' steps, two waves a SIMD (384 entries x 4 heads of 384 x 384, d = 32:
// 95 us; three waves spill and take 340).
constexpr int dbias_waves(int dtype, int d) { return d <= 32 || (d <= 64 && dtype == 1) ? 2 : 1; }

template <typename T, int DP, int KC>
__global__ __launch_bounds__(256, dbias_waves(sizeof(T) == 2 ? 1 : 0, DP)) void k_cross_dbias(const CrossArgs a, int slot_heads, int shared_heads, int shared,
                                                     int qtiles, int ktiles) {
    using TL = Tile<T, DP, KC>;
    constexpr int NB = KC / 32, NS = DP / 16, kPer = 16 / (int)sizeof(T);
    using QL = Tile<T, DP, 32>;
    constexpr int BUF = sizeof(T) == 4 && DP == 128 ? 1 : 2;   // buffers of keys (a second does not fit 160 KB there)
    __shared__ __align__(16) char mem[BUF * 2 * TL::kBytes];
    __shared__ __align__(16) char qmem[4][2 * QL::kBytes];     // a wave's 32 queries: q and dout
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6), ql = lane & 31, hi = lane >> 5;

    uint32_t blk = xcd_block();
    const int kt_ = (int)(blk % (uint32_t)ktiles);
    blk /= (uint32_t)ktiles;
    const int qt_ = (int)(blk % (uint32_t)qtiles);
    blk /= (uint32_t)qtiles;
    const int split = (int)(blk % (uint32_t)a.splits);
    const int64_t slot = blk / (uint32_t)a.splits;
    const int64_t slot_b = slot / slot_heads;
    const int slot_h = (int)(slot - slot_b * slot_heads);
    const int k0 = kt_ * KC, qw = qt_ * 128 + 32 * w;
    const bool wave_live = qw < a.nq, valid = qw + ql < a.nq;
    const int qi = qw + ql;
    const int e0 = (int)((int64_t)shared * split / a.splits), e1 = (int)((int64_t)shared * (split + 1) / a.splits);

    f32x16_t bv[NB], acc[NB];               // the lane's bias, the same for all entries and heads here, and its gradient
    {
        BiasRow<T, KC> bias;
        bias.init(a, slot_b, slot_h, min(qw, a.nq - 1), min(qw + 31, a.nq - 1), min(qw + ql, a.nq - 1), hi);
        bias.load(k0, a.nk);
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const float4 x = bias.get(n, g);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    bv[n][4 * g + e] = f4_get(x, e);
                    acc[n][4 * g + e] = 0.f;
                }
            }
    }

    TL tl;
    tl.init(lane);
    Part<T, DP, KC, 256> kp, vp;
    KeyByte kbyte;
    // q and dout as whole rows, and the fragments through LDS: loaded as fragments, each load would touch 32 rows for
    // 32 bytes of each
    Part<T, DP, 32, 64> qn, gn;
    kp.init(a.k.token, a.d, t);
    vp.init(a.v.token, a.d, t);
    qn.init(a.q.token, a.d, lane);
    gn.init(a.dout.token, a.d, lane);
    float4 row4;
    const int rows_left = max(a.nq - qw, 0), per_key = a.group * a.key_div;
    // the e-th entry and head of those that share this bias, heads innermost
    struct At {
        int64_t b;
        int h;
    };
    auto next = [&](At& at) {
        if (++at.h == slot_h + shared_heads) {
            at.h = slot_h;
            ++at.b;
        }
    };
    auto load_keys = [&](const At& at, bool any) {
        const int hk = at.h / per_key, n = any ? a.nk : 0;
        kp.load((const T*)a.k.data + at.b * a.k.batch + hk * a.k.head, a.k.token, k0, n, a.d);
        vp.load((const T*)a.v.data + at.b * a.v.batch + hk * a.v.head, a.v.token, k0, n, a.d);
        kbyte.load(a.mask && any ? a.mask + at.b * a.mask_batch : nullptr, k0, n, lane);
    };
    auto load_queries = [&](const At& at, bool any) {
        const int n = any ? rows_left : 0;
        qn.load((const T*)a.q.data + at.b * a.q.batch + (int64_t)qw * a.q.token + at.h * a.q.head, a.q.token, 0, n, a.d);
        gn.load((const T*)a.dout.data + at.b * a.dout.batch + (int64_t)qw * a.dout.token + at.h * a.dout.head, a.dout.token, 0, n, a.d);
        row4 = __builtin_bit_cast(float4, buf_load16(make_rsrc(reinterpret_cast<const float4*>(a.rows) + (at.b * a.heads + at.h) * a.nq + qw,
                                                               16u * (uint32_t)min(n, 32)), 16 * ql));
    };
    At at{slot_b + e0 / shared_heads, slot_h + e0 % shared_heads};
    load_keys(at, e0 < e1);
    load_queries(at, e0 < e1);
    for (int e = e0; e < e1; ++e) {
        char* kt = mem + (BUF == 2 ? (e - e0) & 1 : 0) * 2 * TL::kBytes;
        char* vt = kt + TL::kBytes;
        uint64_t bits = kbyte.bits(a.mask, k0, a.nk, lane);
        if (KC == 32) bits &= 0xffffffffull;
        const bool some = bits != (KC == 64 ? ~0ull : 0xffffffffull), more = e + 1 < e1;
        if (BUF == 1) __syncthreads();
        kp.stage(kt, t, some, bits);
        vp.stage(vt, t, some, bits);
        next(at);
        load_keys(at, more);
        const RowStat st{row4.x, row4.y, row4.z, row4.w};
        wave_sync();
        qn.stage(qmem[w], lane, false, 0);
        gn.stage(qmem[w] + QL::kBytes, lane, false, 0);
        load_queries(at, more);
        __syncthreads();
        if (bits != 0 && wave_live) {
            const bool far = __any(st.far());
            f32x16_t s[NB], dp[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = dp[n][r] = 0.f;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                Frag<T> q, f;
                QL::row(qmem[w], ql, hi, i, q);
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    tl.rows(kt, n, i, f);
                    s[n] = mma(f, q, s[n]);
                }
            }
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                Frag<T> g, f;
                QL::row(qmem[w] + QL::kBytes, ql, hi, i, g);
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    tl.rows(vt, n, i, f);
                    dp[n] = mma(f, g, dp[n]);
                }
            }
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = __builtin_fmaf(s[n][r], a.scale, bv[n][r]);
            if (some)
#pragma unroll
                for (int n = 0; n < NB; ++n) drop_absent(s[n], (uint32_t)(bits >> ((KC / 2) * hi + 16 * n)));
            float sh = st.sh;
            if (far) {
#pragma unroll
                for (int n = 0; n < NB; ++n) take_from(s[n], 1.f, st.M);
                sh = st.n2;
            }
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    acc[n][r] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], kLog2e, sh)), dp[n][r] - st.D, acc[n][r]);
        }
    }
    if (!valid) return;
    const int kk = k0 + (KC / 2) * hi;
    if (a.splits > 1) {
        const int64_t ldp = (int64_t)ktiles * KC, slots = gridDim.x / ((int64_t)ktiles * qtiles * a.splits);
        float* po = a.part + (((int64_t)split * slots + slot) * a.nq + qi) * ldp + kk;
#pragma unroll
        for (int j = 0; j < 4 * NB; ++j)
            *reinterpret_cast<float4*>(po + 4 * j) = make_float4(acc[j / 4][4 * (j % 4)], acc[j / 4][4 * (j % 4) + 1],
                                                                 acc[j / 4][4 * (j % 4) + 2], acc[j / 4][4 * (j % 4) + 3]);
        return;
    }
    T* po = (T*)a.dbias.data + slot_b * a.dbias.batch + slot_h * a.dbias.head + (int64_t)qi * a.dbias.row + kk;
#pragma unroll
    for (int j = 0; j < 4 * NB; ++j) {
        const float v[4] = {acc[j / 4][4 * (j % 4)], acc[j / 4][4 * (j % 4) + 1], acc[j / 4][4 * (j % 4) + 2],
                            acc[j / 4][4 * (j % 4) + 3]};
        if (kk + 4 * j + 4 <= a.nk) {
            store4(po + 4 * j, v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (kk + 4 * j + x < a.nk) Store<T>::st(po + 4 * j + x, v[x]);
        }
    }
}

// The splits' sums, 4 keys a thread, in the order of the splits.
template <typename T>
__global__ __launch_bounds__(256) void k_cross_dbias_sum(const CrossArgs a, int slot_heads, int64_t slots, int64_t ldp) {
    const int64_t per_row = (a.nk + 3) / 4, n = slots * a.nq * per_row;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int64_t rowi = i / per_row, slot = rowi / a.nq;
    const int k = (int)(i - rowi * per_row) * 4;
    const float* p = a.part + rowi * ldp + k;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < a.splits; ++s) {
        const float4 y = *reinterpret_cast<const float4*>(p + (int64_t)s * slots * a.nq * ldp);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
    }
    const int64_t slot_b = slot / slot_heads, slot_h = slot - slot_b * slot_heads;
    T* po = (T*)a.dbias.data + slot_b * a.dbias.batch + slot_h * a.dbias.head + (rowi - slot * a.nq) * a.dbias.row + k;
    if (k + 4 <= a.nk) {
        store4(po, x.x, x.y, x.z, x.w);
    } else {
        for (int e = 0; e < a.nk - k; ++e) Store<T>::st(po + e, f4_get(x, e));
    }
}

template <typename T> constexpr int kKeyChunk = sizeof(T) == 2 ? 64 : 32;
int key_chunk(int dtype) { return dtype == 1 ? 64 : 32; }

template <typename T, int DP, bool BIAS, bool DIRECT>
hipError_t backward_q(const CrossArgs& a, hipStream_t s) {
    const int cols = a.nq * a.group;
    const bool solo = cross_solo(a.batch * a.kv_heads, cols), few = !solo && cross_few(a.batch * a.kv_heads, cols);
    const int ctiles = few ? (cols + 31) / 32 : (cols + 127) / 128;
    const dim3 grid((unsigned)(a.batch * a.kv_heads * ctiles));
    constexpr int KC = DP == 128 ? 32 : kKeyChunk<T>;
    if (solo) hipLaunchKernelGGL((k_cross_backward_q<T, DP, 32, 4, true, BIAS, DIRECT>), dim3((grid.x + 3) / 4), dim3(256), 0, s, a, ctiles);
    else if (few) hipLaunchKernelGGL((k_cross_backward_q<T, DP, 32, 4, false, BIAS, DIRECT>), grid, dim3(256), 0, s, a, ctiles);
    else hipLaunchKernelGGL((k_cross_backward_q<T, DP, KC, 1, false, BIAS, DIRECT>), grid, dim3(256), 0, s, a, ctiles);
    return hipGetLastError();
}

// d > 64: in bf16 eight waves to 128 keys; in fp32 a wave's registers do not hold a chunk of its own.
constexpr bool kv_two(int dtype, int d) { return dtype == 1 && d > 64; }
constexpr bool kv_may_be_few(int dtype, int d) { return dtype == 1 || d <= 64; }

template <typename T, int DP, bool BIAS>
hipError_t backward_kv(const CrossArgs& args, const CrossKvPlan& p, hipStream_t s) {
    CrossArgs a = args;
    a.splits = p.splits;
    constexpr int dt = sizeof(T) == 2 ? 1 : 0;
    constexpr bool kTwo = kv_two(dt, DP);
    const int kv_heads = a.kv_heads / a.key_div;
    const dim3 grid((unsigned)(a.batch * kv_heads * p.ktiles * p.splits));
    if constexpr (kv_may_be_few(dt, DP)) {
        if (p.few) hipLaunchKernelGGL((k_cross_backward_kv<T, DP, 32, 4, false, BIAS>), grid, dim3(256), 0, s, a, p.ktiles);
        else hipLaunchKernelGGL((k_cross_backward_kv<T, DP, 32, 1, kTwo, BIAS>), grid, dim3(kTwo ? 512 : 256), 0, s, a, p.ktiles);
    } else {
        hipLaunchKernelGGL((k_cross_backward_kv<T, DP, 32, 1, kTwo, BIAS>), grid, dim3(kTwo ? 512 : 256), 0, s, a, p.ktiles);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const int64_t n = 2 * a.batch * kv_heads * a.nk * a.d / 4;
    hipLaunchKernelGGL((k_cross_kv_sum<T>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a, kv_heads);
    return hipGetLastError();
}

template <typename T, int DP, bool BIAS, bool DIRECT>
hipError_t backward_both(const CrossArgs& args, const CrossKvPlan& p, hipStream_t s) {
    if constexpr (kv_may_be_few(sizeof(T) == 2 ? 1 : 0, DP)) {
        CrossArgs a = args;
        a.splits = 1;
        const int ctiles = (a.nq * a.group + 31) / 32, q_blocks = (int)(a.batch * a.kv_heads) * ctiles;
        hipLaunchKernelGGL((k_cross_rows<T>), dim3((unsigned)((a.batch * a.heads * a.nq + 15) / 16)), dim3(256), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((k_cross_backward_both<T, DP, BIAS, DIRECT>), dim3((unsigned)(q_blocks + (int)(a.batch * (a.kv_heads / a.key_div)) * p.ktiles)),
                           dim3(256), 0, s, a, ctiles, p.ktiles, q_blocks);
        return hipGetLastError();
    } else {
        return hipErrorInvalidValue;        // (cross_both is false)
    }
}

template <typename T, int DP>
hipError_t backward_bias(const CrossArgs& a, hipStream_t s) {
    constexpr int KC = kKeyChunk<T>;
    const int64_t slot_b = a.bias.batch ? a.batch : 1, slot_h = a.bias.head ? a.heads : 1;
    const int shared_heads = a.bias.head ? 1 : a.heads;
    const int shared = (int)((a.bias.batch ? 1 : a.batch) * shared_heads);
    const int qtiles = (a.nq + 127) / 128, ktiles = (a.nk + KC - 1) / KC;
    const dim3 grid((unsigned)(slot_b * slot_h * a.splits * qtiles * ktiles));
    hipLaunchKernelGGL((k_cross_dbias<T, DP, KC>), grid, dim3(256), 0, s, a, (int)slot_h, shared_heads, shared, qtiles, ktiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int64_t n = slot_b * slot_h * a.nq * ((a.nk + 3) / 4);
    hipLaunchKernelGGL((k_cross_dbias_sum<T>), dim3((unsigned)((n + 255) / 256)), dim3(256), 0, s, a, (int)slot_h,
                       slot_b * slot_h, (int64_t)ktiles * KC);
    return hipGetLastError();
}

}  // namespace

// Tiles of 128 keys from one for each compute unit on (half a one where eight
// waves share a tile), else of 32.  The queries are split where that fills the
// compute units better: an estimate of the time, the ten operations a score and
// channel at the rate that the pass reaches on a full chip over the share of it
// that the work-groups keep busy, plus the sums' launch and their bytes.  A split
// keeps 16 chunks of 32 queries.  (2 entries x 4 key heads of 3000 keys, d = 128:
// 192 work-groups, one to a compute unit, 367 us; 768 in four splits, 303 and 18 us.)
CrossKvPlan cross_kv_plan(int dtype, int d, int64_t heads, int64_t nk, int64_t per_head, int64_t group) {
    CrossKvPlan p{false, 0, 1};
    const bool two = kv_two(dtype, d);
    const int64_t wide = (nk + 127) / 128;
    p.few = kv_may_be_few(dtype, d) && heads * wide < (two ? 128 : 256);
    p.ktiles = (int)(p.few ? (nk + 31) / 32 : wide);
    const int64_t groups = heads * p.ktiles, chunks = (per_head + 31) / 32 * group;
    if (groups < 1 || chunks < 1) return p;
    const double places = 256.0 * (two && !p.few ? 1 : d <= 32 && dtype == 1 ? 3 : d <= 64 ? 2 : 1);
    const double work = 10.0 * (double)heads * (double)nk * (double)per_head * (double)group * d / (dtype == 1 ? 500e6 : 60e6);   // us
    const double bytes = 2.0 * (double)heads * (double)nk * d * 4;
    double best = 0;
    for (int n = 1; n <= 16 && n * 16 <= std::max<int64_t>(chunks, 16); ++n) {
        const double busy = (double)groups * n / places, t = work * std::ceil(busy) / busy + (n > 1 ? 8 + 2 * n * bytes / 4e6 : 0);
        if (n == 1 || t < 0.95 * best) {
            best = t;
            p.splits = n;
        }
    }
    return p;
}

// Both passes side by side where their work-groups of 32 columns and of 32 keys together
// are one to a compute unit at most.  (300 x 500, 8 heads of 64 with a bias, fp32, 80 + 128: 25 and
// 23 us one after the other, 26 together and 4 for the rows before; 512 x 512, bf16,
// 128 + 128: 12.5 and 10.7, 13.2 and 4.  With more they take turns on the compute units: 200 x 2000, 8
// heads of 32, 56 + 504: 19.6 and 8.0, 32.9 and 3.7.)
bool cross_both(const CrossArgs& a, const CrossKvPlan& p) {
    const int64_t heads = a.batch * a.kv_heads, cols = (int64_t)a.nq * a.group;
    return p.few && p.splits == 1 && a.nq > 0 && cross_few(heads, cols) && !cross_solo(heads, cols) &&
           heads * ((cols + 31) / 32) + a.batch * (a.kv_heads / a.key_div) * p.ktiles <= 256;
}

size_t cross_kv_part_floats(const CrossKvPlan& p, int64_t heads, int64_t nk, int d) {
    return p.splits > 1 ? (size_t)p.splits * 2 * (size_t)heads * (size_t)nk * (size_t)d : 0;
}

// The entries and heads of a bias are split where that shortens the pass: its
// rounds of work-groups (two to a compute unit, or one) times the entries that each
// of them takes, against the sums' launch and the bytes of the partial sums, in
// entries' times.  A split keeps four.  (384 entries, 72 tiles, d = 32: seven splits,
// 504 work-groups, 100 us and 5 for the sums; fifteen, 1080, 116 and 7; 28, 2016, 112 and 11.)
int cross_dbias_splits(int dtype, int d, int64_t slots, int64_t shared, int64_t nq, int64_t nk) {
    const int kc = key_chunk(dtype);
    const int64_t tiles = slots * ((nq + 127) / 128) * ((nk + kc - 1) / kc), places = dbias_waves(dtype, d) * 256;
    if (tiles < 1 || tiles >= 4 * places) return 1;
    int64_t best_n = 1;
    double best = 0;
    for (int rounds = 0; rounds <= 4; ++rounds) {              // one split, and the most that rounds of work-groups hold
        const int64_t n = rounds ? std::min(rounds * places / tiles, shared / 4) : 1;
        if (n < 1) continue;
        const double t = (double)((tiles * n + places - 1) / places * ((shared + n - 1) / n)) + (n > 1 ? 2 + 0.01 * (double)(n * tiles) : 0);
        if (rounds == 0 || t < 0.97 * best) {
            best = t;
            best_n = n;
        }
    }
    return (int)best_n;
}

size_t cross_dbias_part_floats(int dtype, int splits, int64_t slots, int64_t nq, int64_t nk) {
    const int kc = key_chunk(dtype);
    return splits > 1 ? (size_t)splits * (size_t)slots * (size_t)nq * (size_t)((nk + kc - 1) / kc * kc) : 0;
}

#define CROSS_BY_TYPE(F)                                                                                        \
    (dtype == 1 ? (a.d <= 32 ? F(bf16_t, 32) : a.d <= 64 ? F(bf16_t, 64) : F(bf16_t, 128))                        \
                : (a.d <= 32 ? F(float, 32) : a.d <= 64 ? F(float, 64) : F(float, 128)))
#define CROSS_Q(T, DP)                                                       \
    (!a.bias.data ? backward_q<T, DP, false, false>(a, s)                    \
                  : a.direct_bias ? backward_q<T, DP, true, true>(a, s) : backward_q<T, DP, true, false>(a, s))
#define CROSS_KV(T, DP) (a.bias.data ? backward_kv<T, DP, true>(a, p, s) : backward_kv<T, DP, false>(a, p, s))
#define CROSS_BIAS(T, DP) (backward_bias<T, DP>(a, s))

#define CROSS_BOTH(T, DP)                                                    \
    (!a.bias.data ? backward_both<T, DP, false, false>(a, p, s)              \
                  : a.direct_bias ? backward_both<T, DP, true, true>(a, p, s) : backward_both<T, DP, true, false>(a, p, s))

hipError_t launch_cross_backward_both(int dtype, const CrossArgs& a, const CrossKvPlan& p, hipStream_t s) { return CROSS_BY_TYPE(CROSS_BOTH); }
hipError_t launch_cross_backward_q(int dtype, const CrossArgs& a, hipStream_t s) { return CROSS_BY_TYPE(CROSS_Q); }
hipError_t launch_cross_backward_kv(int dtype, const CrossArgs& a, const CrossKvPlan& p, hipStream_t s) { return CROSS_BY_TYPE(CROSS_KV); }
hipError_t launch_cross_backward_bias(int dtype, const CrossArgs& a, hipStream_t s) { return CROSS_BY_TYPE(CROSS_BIAS); }

}  // namespace trimul
