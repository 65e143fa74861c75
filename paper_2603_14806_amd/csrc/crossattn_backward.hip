// Attention of queries over keys of another length, backward.  From the
// forward's M_i and L_i the weights are P_ij = exp(x_ij - M_i) / L_i again, and
//
//     D_i = dout_i . out_i        dS_ij = P_ij (dout_i . v_j - D_i)
//     dq_i = scale sum_j dS_ij k_j        dbias = dS, summed where a bias is shared
//     dk_j = scale sum_i dS_ij q_i        dv_j = sum_i P_ij dout_i
//
// Three passes, each the owner of what it writes, so that every sum has one
// order and nothing is added atomically: queries (dq, and D for the others),
// keys (dk, dv; a key head's loop runs over the columns of all its query
// heads) and, where a bias is given, tiles of it (whose loop runs over the
// entries and heads that share it).  Each recomputes S and dP.
#include "crossattn.h"

namespace trimul {
namespace {

template <typename T>
__device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
    if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
    else *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
}

// A query's statistics as the weights use them: P = exp2((x - M) log2 e + n2) = exp2(x log2 e + sh).
// A query with no key: M = 0, n2 = -inf, P = 0.
struct RowStat {
    float M, n2, sh;
    __device__ __forceinline__ void set(float m, float l) {
        M = l == 0.f ? 0.f : m;
        n2 = l == 0.f ? -INFINITY : -__builtin_amdgcn_logf(l);
        sh = __builtin_fmaf(-M, kLog2e, n2);
    }
    __device__ __forceinline__ bool far() const { return !(fabsf(M * kLog2e) <= kFmaMax); }
};

// P of one score: s = q . k, bv its bias.
template <bool BIAS, bool FAR>
__device__ __forceinline__ float weight(float s, float bv, float scale, float coef, float M, float n2, float sh) {
    if (FAR) {
        const float x = BIAS ? __builtin_fmaf(s, scale, bv) : s * scale;
        return __builtin_amdgcn_exp2f(__builtin_fmaf(x - M, kLog2e, n2));
    }
    const float x = BIAS ? __builtin_fmaf(s, scale, bv) : s;
    return __builtin_amdgcn_exp2f(__builtin_fmaf(x, coef, sh));
}

// ------------------------------------------------------------------ queries: dq, D
//
// The forward's layout (lane: one column, registers: keys), 32 columns a wave.
template <typename T, int DP, int KC, bool BIAS>
__global__ __launch_bounds__(256) void k_cross_backward_q(const CrossArgs a, int ctiles) {
    using TL = Tile<T, DP, KC>;
    constexpr int NB = KC / 32, ND = DP / 32, NS = DP / 16;
    __shared__ __align__(16) char mem[2 * 2 * TL::kBytes];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, ql = lane & 31, hi = lane >> 5;

    int64_t blk = blockIdx.x;
    const int ct = (int)(blk % ctiles);
    blk /= ctiles;
    const int hk = (int)(blk % a.kv_heads);
    const int64_t b = blk / a.kv_heads;
    const int ncols = a.nq * a.group, cw = ct * 128 + 32 * w;
    const bool wave_live = cw < ncols, valid = cw + ql < ncols;
    const int col = min(cw + ql, ncols - 1);
    const int qi = col / a.group, h = hk * a.group + (col - qi * a.group);
    const int64_t row = (b * a.heads + h) * a.nq + qi;

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
        }
        D += xor32(D);
        if (valid && !hi) a.delta[row] = D;
    }
    RowStat st;
    st.set(a.stats[row], a.stats[a.batch * a.heads * a.nq + row]);
    const bool far = __any(st.far());
    const float coef = BIAS ? kLog2e : a.scale * kLog2e;
    const T* kb = (const T*)a.k.data + b * a.k.batch + hk * a.k.head;
    const T* vb = (const T*)a.v.data + b * a.v.batch + hk * a.v.head;
    const T* brow = BIAS ? (const T*)a.bias.data + b * a.bias.batch + h * a.bias.head + (int64_t)qi * a.bias.row : nullptr;
    const uint8_t* mask = a.mask ? a.mask + b * a.mask_batch : nullptr;
    const int nchunks = (a.nk + KC - 1) / KC;

    f32x16_t acc[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] = 0.f;

    Part<T, DP, KC, 256> kp, vp;
    KeyByte kbyte;
    BiasRow<T, KC> bp;
    auto load = [&](int c) {
        kp.load(kb, a.k.token, c * KC, a.nk, a.d, t);
        vp.load(vb, a.v.token, c * KC, a.nk, a.d, t);
        kbyte.load(mask, c * KC, a.nk, lane);
    };
    if (nchunks) {
        load(0);
        if (BIAS) bp.load(brow, (KC / 2) * hi, a.nk);
    }
    for (int c = 0; c < nchunks; ++c) {
        char* kt = mem + (c & 1) * 2 * TL::kBytes;
        char* vt = kt + TL::kBytes;
        uint64_t bits = kbyte.bits(c * KC, a.nk, lane);
        if (KC == 32) bits &= 0xffffffffull;
        const bool some = bits != (KC == 64 ? ~0ull : 0xffffffffull);
        kp.stage(kt, t, some, bits);
        vp.stage(vt, t, some, bits);
        if (c + 1 < nchunks) load(c + 1);
        __syncthreads();
        if (bits != 0 && wave_live) {
            const uint32_t mine = (uint32_t)(bits >> ((KC / 2) * hi));
            f32x16_t s[NB], dp[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = dp[n][r] = 0.f;
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    Frag<T> f;
                    TL::rows(kt, lane, n, i, f);
                    s[n] = mma(f, qf[i], s[n]);
                }
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    Frag<T> f;
                    TL::rows(vt, lane, n, i, f);
                    dp[n] = mma(f, gf[i], dp[n]);
                }
            }
            auto grads = [&](auto masked, auto isfar) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        float4 bv = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (BIAS) bv = bp.get(n, g);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int r = 4 * g + e;
                            float p = weight<BIAS, decltype(isfar)::value>(s[n][r], f4_get(bv, e), a.scale, coef, st.M, st.n2, st.sh);
                            if (decltype(masked)::value) p = (mine >> (16 * n + r)) & 1 ? p : 0.f;
                            s[n][r] = p * (dp[n][r] - D);
                        }
                    }
            };
            if (far) grads(std::true_type{}, std::true_type{});
            else if (some) grads(std::true_type{}, std::false_type{});
            else grads(std::false_type{}, std::false_type{});
            if (BIAS && c + 1 < nchunks) bp.load(brow, (c + 1) * KC + (KC / 2) * hi, a.nk);
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) {
                    Frag<T> pf;
                    take8(s[n], tt, pf);
#pragma unroll
                    for (int i = 0; i < ND; ++i) {
                        Frag<T> kf;
                        TL::cols(kt, lane, n, tt, i, kf);
                        acc[i] = mma(kf, pf, acc[i]);
                    }
                }
        } else if (BIAS && c + 1 < nchunks) {
            bp.load(brow, (c + 1) * KC + (KC / 2) * hi, a.nk);
        }
    }
    if (!valid) return;
    T* po = (T*)a.dq.data + b * a.dq.batch + (int64_t)qi * a.dq.token + h * a.dq.head;
#pragma unroll
    for (int j = 0; j < 4 * ND; ++j) {
        const int c = 8 * j + 4 * hi;
        if (c < a.d)
            store4(po + c, acc[j / 4][4 * (j % 4)] * a.scale, acc[j / 4][4 * (j % 4) + 1] * a.scale,
                   acc[j / 4][4 * (j % 4) + 2] * a.scale, acc[j / 4][4 * (j % 4) + 3] * a.scale);
    }
}

// ------------------------------------------------------------------ keys: dk, dv
//
// Lane: one key (K and V as B operands in registers), registers: the queries of
// a chunk of QC columns, whose q and dout pass through LDS; 32 keys a wave.
// The bias tile of a chunk passes through LDS too and is read transposed
// (four queries of one key at a time).
template <typename T, int DP, int QC, bool BIAS>
__global__ __launch_bounds__(256) void k_cross_backward_kv(const CrossArgs a, int ktiles) {
    using TL = Tile<T, DP, QC>;
    constexpr int NB = QC / 32, ND = DP / 32, NS = DP / 16, kN = QC * TL::kPieces / 256;
    constexpr int kBRow = 128 * (int)sizeof(T) + (sizeof(T) == 2 ? 64 : 16);   // spreads four rows over the banks
    constexpr int kBPieces = 128 * (int)sizeof(T) / 16, kBN = QC * kBPieces / 256;
    __shared__ __align__(16) char mem[2 * 2 * TL::kBytes];
    __shared__ __align__(16) char bmem[BIAS ? 2 * QC * kBRow : 16];
    __shared__ __align__(16) float stat[2][4][QC];             // M, n2, sh, D of a chunk's columns
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, kl = lane & 31, hi = lane >> 5;

    int64_t blk = blockIdx.x;
    const int kt_ = (int)(blk % ktiles);
    blk /= ktiles;
    const int hk = (int)(blk % a.kv_heads);
    const int64_t b = blk / a.kv_heads;
    const int key0 = kt_ * 128, key = key0 + 32 * w + kl;
    const bool valid = key < a.nk, wave_live = key0 + 32 * w < a.nk;
    const int kc = min(key, a.nk - 1);
    const bool present = valid && (!a.mask || a.mask[b * a.mask_batch + kc] != 0);
    const bool all_present = __all(present);
    const int ncols = a.nq * a.group, nchunks = (ncols + QC - 1) / QC;
    const float coef = BIAS ? kLog2e : a.scale * kLog2e;

    Frag<T> kf[NS], vf[NS];
    {
        const T* kr = (const T*)a.k.data + b * a.k.batch + (int64_t)kc * a.k.token + hk * a.k.head;
        const T* vr = (const T*)a.v.data + b * a.v.batch + (int64_t)kc * a.v.token + hk * a.v.head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            load_row(kr, s, hi, a.d, kf[s]);
            load_row(vr, s, hi, a.d, vf[s]);
        }
    }
    f32x16_t dk[ND], dv[ND];
#pragma unroll
    for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) dk[i][r] = dv[i][r] = 0.f;

    uint4 qp[kN], gp[kN], bp[BIAS ? kBN : 1];
    float sm = 0.f, sl = 0.f, sd = 0.f;
    const T* qb = (const T*)a.q.data + b * a.q.batch;
    const T* gb = (const T*)a.dout.data + b * a.dout.batch;
    const int64_t rows = a.batch * a.heads * a.nq;
    auto split_col = [&](int c, int& qi, int& h) {
        qi = a.group == 1 ? c : c / a.group;
        h = hk * a.group + (c - qi * a.group);
    };
    auto load = [&](int c) {
        int qi, h;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int u = t + 256 * i, piece = u % TL::kPieces;
            split_col(min(c * QC + u / TL::kPieces, ncols - 1), qi, h);
            const int ch = piece * TL::kPer < a.d ? piece * TL::kPer : 0;
            qp[i] = *reinterpret_cast<const uint4*>(qb + (int64_t)qi * a.q.token + h * a.q.head + ch);
            gp[i] = *reinterpret_cast<const uint4*>(gb + (int64_t)qi * a.dout.token + h * a.dout.head + ch);
        }
        if (BIAS)
#pragma unroll
            for (int i = 0; i < kBN; ++i) {
                const int u = t + 256 * i, k = key0 + (u % kBPieces) * TL::kPer;
                split_col(min(c * QC + u / kBPieces, ncols - 1), qi, h);
                bp[i] = *reinterpret_cast<const uint4*>((const T*)a.bias.data + b * a.bias.batch + h * a.bias.head +
                                                        (int64_t)qi * a.bias.row + (k < a.nk ? k : 0));
            }
        const int cc = c * QC + (lane & (QC - 1));
        split_col(min(cc, ncols - 1), qi, h);
        const int64_t row = (b * a.heads + h) * a.nq + qi;
        sm = a.stats[row];
        sl = cc < ncols ? a.stats[rows + row] : 0.f;           // columns past the last have weight 0
        sd = a.delta[row];
    };
    if (nchunks) load(0);
    for (int c = 0; c < nchunks; ++c) {
        const int buf = c & 1;
        char* qt = mem + buf * 2 * TL::kBytes;
        char* gt = qt + TL::kBytes;
        char* bt = bmem + (BIAS ? buf * QC * kBRow : 0);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int u = t + 256 * i;
            const uint32_t off = TL::off(u / TL::kPieces, u % TL::kPieces);
            *reinterpret_cast<uint4*>(qt + off) = qp[i];
            *reinterpret_cast<uint4*>(gt + off) = gp[i];
        }
        if (BIAS)
#pragma unroll
            for (int i = 0; i < kBN; ++i) {
                const int u = t + 256 * i;
                *reinterpret_cast<uint4*>(bt + (u / kBPieces) * kBRow + (u % kBPieces) * 16) = bp[i];
            }
        RowStat st;
        st.set(sm, sl);
        const bool far = __any(st.far());
        if (w == 0 && lane < QC) {
            stat[buf][0][lane] = st.M;
            stat[buf][1][lane] = st.n2;
            stat[buf][2][lane] = st.sh;
            stat[buf][3][lane] = sd;
        }
        if (c + 1 < nchunks) load(c + 1);
        __syncthreads();
        if (!wave_live) continue;
        f32x16_t s[NB], dp[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[n][r] = dp[n][r] = 0.f;
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                Frag<T> f;
                TL::rows(qt, lane, n, i, f);
                s[n] = mma(f, kf[i], s[n]);
            }
#pragma unroll
            for (int i = 0; i < NS; ++i) {
                Frag<T> f;
                TL::rows(gt, lane, n, i, f);
                dp[n] = mma(f, vf[i], dp[n]);
            }
        }
        auto grads = [&](auto masked, auto isfar) {
            constexpr bool FAR = decltype(isfar)::value;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int r0 = (QC / 2) * hi + 16 * n + 4 * g;      // the lane's four tile rows
                    float4 bv = make_float4(0.f, 0.f, 0.f, 0.f);
                    if constexpr (BIAS) {
                        if constexpr (sizeof(T) == 2) {
                            const uint2 x = lds_tr4(bt + (r0 + ((lane >> 2) & 3)) * kBRow +
                                                    (32 * w + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)) * 2);
                            bv = bf4(x.x, x.y);
                        } else {
                            const char* p = bt + r0 * kBRow + (32 * w + kl) * 4;
                            bv = make_float4(*(const float*)p, *(const float*)(p + kBRow), *(const float*)(p + 2 * kBRow),
                                             *(const float*)(p + 3 * kBRow));
                        }
                    }
                    const float4 d4 = *reinterpret_cast<const float4*>(&stat[buf][3][r0]);
                    float4 m4, n4, h4;
                    if (FAR) {
                        m4 = *reinterpret_cast<const float4*>(&stat[buf][0][r0]);
                        n4 = *reinterpret_cast<const float4*>(&stat[buf][1][r0]);
                    } else {
                        h4 = *reinterpret_cast<const float4*>(&stat[buf][2][r0]);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int r = 4 * g + e;
                        float p = weight<BIAS, FAR>(s[n][r], f4_get(bv, e), a.scale, coef, FAR ? f4_get(m4, e) : 0.f,
                                                    FAR ? f4_get(n4, e) : 0.f, FAR ? 0.f : f4_get(h4, e));
                        float ds = p * (dp[n][r] - f4_get(d4, e));
                        if (decltype(masked)::value) {          // an absent key's k and v may hold anything
                            p = present ? p : 0.f;
                            ds = present ? ds : 0.f;
                        }
                        s[n][r] = p;
                        dp[n][r] = ds;
                    }
                }
        };
        if (far) grads(std::true_type{}, std::true_type{});
        else if (!all_present) grads(std::true_type{}, std::false_type{});
        else grads(std::false_type{}, std::false_type{});
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                Frag<T> pf, df;
                take8(s[n], tt, pf);
                take8(dp[n], tt, df);
#pragma unroll
                for (int i = 0; i < ND; ++i) {
                    Frag<T> f;
                    TL::cols(gt, lane, n, tt, i, f);
                    dv[i] = mma(f, pf, dv[i]);
                    TL::cols(qt, lane, n, tt, i, f);
                    dk[i] = mma(f, df, dk[i]);
                }
            }
    }
    if (!valid) return;
    T* pk = (T*)a.dk.data + b * a.dk.batch + (int64_t)key * a.dk.token + hk * a.dk.head;
    T* pv = (T*)a.dv.data + b * a.dv.batch + (int64_t)key * a.dv.token + hk * a.dv.head;
#pragma unroll
    for (int j = 0; j < 4 * ND; ++j) {
        const int c = 8 * j + 4 * hi;
        if (c < a.d) {
            store4(pk + c, dk[j / 4][4 * (j % 4)] * a.scale, dk[j / 4][4 * (j % 4) + 1] * a.scale,
                   dk[j / 4][4 * (j % 4) + 2] * a.scale, dk[j / 4][4 * (j % 4) + 3] * a.scale);
            store4(pv + c, dv[j / 4][4 * (j % 4)], dv[j / 4][4 * (j % 4) + 1], dv[j / 4][4 * (j % 4) + 2],
                   dv[j / 4][4 * (j % 4) + 3]);
        }
    }
}

// ------------------------------------------------------------------ dbias
//
// One work-group: 128 queries x KC keys of one bias (the query pass's layout), its loop over the
// entries and heads that share the bias (a split of them: the sums of the splits are added by
// k_cross_dbias_sum).
template <typename T, int DP, int KC>
__global__ __launch_bounds__(256) void k_cross_dbias(const CrossArgs a, int slot_heads, int shared_heads, int shared,
                                                     int qtiles, int ktiles) {
    using TL = Tile<T, DP, KC>;
    constexpr int NB = KC / 32, NS = DP / 16, kPer = 16 / (int)sizeof(T);
    __shared__ __align__(16) char mem[2 * 2 * TL::kBytes];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, ql = lane & 31, hi = lane >> 5;

    int64_t blk = blockIdx.x;
    const int kt_ = (int)(blk % ktiles);
    blk /= ktiles;
    const int qt_ = (int)(blk % qtiles);
    blk /= qtiles;
    const int split = (int)(blk % a.splits);
    const int64_t slot = blk / a.splits;
    const int64_t slot_b = slot / slot_heads;
    const int slot_h = (int)(slot - slot_b * slot_heads);
    const int k0 = kt_ * KC, qw = qt_ * 128 + 32 * w;
    const bool wave_live = qw < a.nq, valid = qw + ql < a.nq;
    const int qi = min(qw + ql, a.nq - 1);
    const int e0 = (int)((int64_t)shared * split / a.splits), e1 = (int)((int64_t)shared * (split + 1) / a.splits);

    BiasRow<T, KC> bias;
    bias.load((const T*)a.bias.data + slot_b * a.bias.batch + slot_h * a.bias.head + (int64_t)qi * a.bias.row,
              k0 + (KC / 2) * hi, a.nk);
    f32x16_t acc[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[n][r] = 0.f;

    Part<T, DP, KC, 256> kp, vp;
    KeyByte kbyte;
    Frag<T> qf[NS], gf[NS];
    float sm, sl, D;
    const int64_t rows = a.batch * a.heads * a.nq;
    // entry and head of the e-th of those that share this bias: heads innermost
    auto load_keys = [&](int e) {
        const int64_t b = slot_b + e / shared_heads;
        const int hk = (slot_h + e % shared_heads) / a.group;
        kp.load((const T*)a.k.data + b * a.k.batch + hk * a.k.head, a.k.token, k0, a.nk, a.d, t);
        vp.load((const T*)a.v.data + b * a.v.batch + hk * a.v.head, a.v.token, k0, a.nk, a.d, t);
        kbyte.load(a.mask ? a.mask + b * a.mask_batch : nullptr, k0, a.nk, lane);
    };
    auto load_queries = [&](int e) {
        const int64_t b = slot_b + e / shared_heads;
        const int h = slot_h + e % shared_heads;
        const T* qr = (const T*)a.q.data + b * a.q.batch + (int64_t)qi * a.q.token + h * a.q.head;
        const T* gr = (const T*)a.dout.data + b * a.dout.batch + (int64_t)qi * a.dout.token + h * a.dout.head;
#pragma unroll
        for (int s = 0; s < NS; ++s) {
            load_row(qr, s, hi, a.d, qf[s]);
            load_row(gr, s, hi, a.d, gf[s]);
        }
        const int64_t row = (b * a.heads + h) * a.nq + qi;
        sm = a.stats[row];
        sl = a.stats[rows + row];
        D = a.delta[row];
    };
    if (e0 < e1) {
        load_keys(e0);
        load_queries(e0);
    }
    for (int e = e0; e < e1; ++e) {
        char* kt = mem + ((e - e0) & 1) * 2 * TL::kBytes;
        char* vt = kt + TL::kBytes;
        uint64_t bits = kbyte.bits(k0, a.nk, lane);
        if (KC == 32) bits &= 0xffffffffull;
        const bool some = bits != (KC == 64 ? ~0ull : 0xffffffffull);
        kp.stage(kt, t, some, bits);
        vp.stage(vt, t, some, bits);
        if (e + 1 < e1) load_keys(e + 1);
        __syncthreads();
        if (bits != 0 && wave_live) {
            const uint32_t mine = (uint32_t)(bits >> ((KC / 2) * hi));
            RowStat st;
            st.set(sm, sl);
            const bool far = __any(st.far());
            const float Dn = D;
            f32x16_t s[NB], dp[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = dp[n][r] = 0.f;
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    Frag<T> f;
                    TL::rows(kt, lane, n, i, f);
                    s[n] = mma(f, qf[i], s[n]);
                }
#pragma unroll
                for (int i = 0; i < NS; ++i) {
                    Frag<T> f;
                    TL::rows(vt, lane, n, i, f);
                    dp[n] = mma(f, gf[i], dp[n]);
                }
            }
            if (e + 1 < e1) load_queries(e + 1);
            auto grads = [&](auto masked, auto isfar) {
#pragma unroll
                for (int n = 0; n < NB; ++n)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float4 bv = bias.get(n, g);
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int r = 4 * g + x;
                            float p = weight<true, decltype(isfar)::value>(s[n][r], f4_get(bv, x), a.scale, kLog2e, st.M, st.n2, st.sh);
                            float ds = p * (dp[n][r] - Dn);
                            if (decltype(masked)::value) ds = (mine >> (16 * n + r)) & 1 ? ds : 0.f;
                            acc[n][r] += ds;
                        }
                    }
            };
            if (far) grads(std::true_type{}, std::true_type{});
            else if (some) grads(std::true_type{}, std::false_type{});
            else grads(std::false_type{}, std::false_type{});
        } else if (e + 1 < e1) {
            load_queries(e + 1);
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

template <typename T, int DP, bool BIAS>
hipError_t backward_q(const CrossArgs& a, hipStream_t s) {
    const int ctiles = (a.nq * a.group + 127) / 128;
    const dim3 grid((unsigned)(a.batch * a.kv_heads * ctiles));
    hipLaunchKernelGGL((k_cross_backward_q<T, DP, kKeyChunk<T>, BIAS>), grid, dim3(256), 0, s, a, ctiles);
    return hipGetLastError();
}

template <typename T, int DP, bool BIAS>
hipError_t backward_kv(const CrossArgs& a, hipStream_t s) {
    const int ktiles = (a.nk + 127) / 128;
    const dim3 grid((unsigned)(a.batch * a.kv_heads * ktiles));
    constexpr int QC = sizeof(T) == 2 && DP == 32 ? 64 : 32;
    hipLaunchKernelGGL((k_cross_backward_kv<T, DP, QC, BIAS>), grid, dim3(256), 0, s, a, ktiles);
    return hipGetLastError();
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

// The work-groups of the tiles alone leave compute units idle below about
// 1024; a split keeps four entries or heads.
int cross_dbias_splits(int dtype, int64_t slots, int64_t shared, int64_t nq, int64_t nk) {
    const int kc = key_chunk(dtype);
    const int64_t tiles = slots * ((nq + 127) / 128) * ((nk + kc - 1) / kc);
    if (tiles < 1 || tiles >= 1024) return 1;
    int64_t n = (1024 + tiles - 1) / tiles;
    if (n > shared / 4) n = shared / 4;
    return n < 1 ? 1 : (int)n;
}

size_t cross_dbias_part_floats(int dtype, int splits, int64_t slots, int64_t nq, int64_t nk) {
    const int kc = key_chunk(dtype);
    return splits > 1 ? (size_t)splits * (size_t)slots * (size_t)nq * (size_t)((nk + kc - 1) / kc * kc) : 0;
}

#define CROSS_BY_TYPE(F)                                                                                        \
    (dtype == 1 ? (a.d <= 32 ? F(bf16_t, 32) : a.d <= 64 ? F(bf16_t, 64) : F(bf16_t, 128))                        \
                : (a.d <= 32 ? F(float, 32) : a.d <= 64 ? F(float, 64) : F(float, 128)))
#define CROSS_Q(T, DP) (a.bias.data ? backward_q<T, DP, true>(a, s) : backward_q<T, DP, false>(a, s))
#define CROSS_KV(T, DP) (a.bias.data ? backward_kv<T, DP, true>(a, s) : backward_kv<T, DP, false>(a, s))
#define CROSS_BIAS(T, DP) (backward_bias<T, DP>(a, s))

hipError_t launch_cross_backward_q(int dtype, const CrossArgs& a, hipStream_t s) { return CROSS_BY_TYPE(CROSS_Q); }
hipError_t launch_cross_backward_kv(int dtype, const CrossArgs& a, hipStream_t s) { return CROSS_BY_TYPE(CROSS_KV); }
hipError_t launch_cross_backward_bias(int dtype, const CrossArgs& a, hipStream_t s) { return CROSS_BY_TYPE(CROSS_BIAS); }

}  // namespace trimul
