// Attention, backward: the probabilities are formed again from the scores and the logarithm of their sum (see mrf_attention_backward in the header).
//
// Two launches, each with its sums in registers from the first tile to the last, so that none depends on what other workgroups do:
//   queries  a workgroup has 128 queries of a head and goes through their keys:   scores, dP, dq.  It also sums dS over the keys, which is 0 but
//            for the rounding of `out` in delta = sum(dout out): what it is not 0, r, is taken off delta, which is then good to 32 bits, and, times
//            sum(P k), off dq (without that, dq in 16 bits was 1.8 times as far off as its own rounding makes it).
//   keys     a workgroup has 128 keys of a head of keys and goes through the queries of all heads that share it:  scores, dP, dv, dk; and, for the table's
//            gradient, sums of dS down the diagonals (below).
// Five products would do; the scores and dP are formed twice, which spares sums over workgroups in an order that changes.
//
// What bounds it: matrix units and LDS, with what a wavefront does between its products beside them only where two or three share a SIMD (heads of 128 have the registers of
// one).  4 sequences of 2,048, 16 heads, without a mask, queries / keys in us: heads of 32 107 / 132, 64 194 / 223 (four products each: 710 / 620 TFLOP/s), 128 338 / 412
// (810 / 670); 64 in 32 bits 850 / 1,470.  With a bias and its table's gradient heads of 64 take 200 / 295.
#include "mrfmp_attention.h"

#include <type_traits>

template <class T> constexpr int mrf_attn_bwd_rows() { return sizeof(T) == 4 ? 32 : 64; }

template <class F> struct MrfTwo { F a, b; };

// steps whose operands are read ahead together (of 128 entries, 4 sequences of 2,048, 16 heads: two 338 and 412 us, four 342 and 420, eight 344 and 423)
template <class T, int DP> constexpr int mrf_attn_group() { return sizeof(T) == 4 ? 1 : 2; }

// ---- dq, and delta
template <class T, int DP, bool BIAS>
__global__ void __launch_bounds__(256, (sizeof(T) == 4 || DP == 128 ? 1 : 2)) mrf_attn_bwd_queries(const MrfAttnParams P)
{
    constexpr int KT = mrf_attn_bwd_rows<T>(), NT = 256, ROWS = 128, LINE = ROWS + KT;
    typedef MrfRows<T, DP, KT, NT> Rows;
    typedef typename MrfFrag<T>::type frag;
    constexpr int TILE = KT * Rows::LD, U = KT / 32, STEPS = DP / 16;
    __shared__ __align__(16) T lds[2][2][TILE];      // keys, values
    __shared__ MrfLine<BIAS ? LINE : 1> line;
    MrfPlaces<T, DP, Rows::LD> places;
    places.template init<Rows>();
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5;
    // (the longest rows of causal ones first)
    const int blocks = (P.Q + ROWS - 1) / ROWS, bh = blockIdx.x % (P.B * P.Hq), block = blocks - 1 - (int)(blockIdx.x / (P.B * P.Hq));
    const int b = bh / P.Hq, h = bh % P.Hq, hk = h / P.G;
    const MrfAttnBatch s(P, b);
    const int r0 = block * ROWS, i = r0 + wv * 32 + (lane & 31);
    const bool there = i < s.nq;
    const int i1 = min(r0 + ROWS - 1, s.nq - 1), w0 = r0 + wv * 32, w1 = min(w0 + 31, s.nq - 1);
    const long long row = (((long long)b * P.Q + i) * P.Hq + h) * P.D, stat = ((long long)b * P.Hq + h) * P.Q + i;

    frag qf[DP / 16] = {}, gf[DP / 16] = {};
    float delta = 0.0f;
    if (w0 <= w1) {
        const int at = min(i, w1);
        const long long dense = (((long long)b * P.Q + at) * P.Hq + h) * P.D;
        const T *q = (const T *)P.q + b * P.qs[0] + at * P.qs[1] + h * P.qs[2], *g = (const T *)P.dout + dense, *o = (const T *)P.out + dense;
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) {
            const int d = 16 * t + 8 * half;
            qf[t] = mrf_load8(q, d, P.D, there);
            gf[t] = mrf_load8(g, d, P.D, there);
            const frag of = mrf_load8(o, d, P.D, there);
#pragma unroll
            for (int j = 0; j < 8; ++j) delta = fmaf(mrf_to_f32((T)gf[t][j]), mrf_to_f32((T)of[j]), delta);
        }
        delta = mrf_halves_sum(delta);
    }
    // a query without keys has no probabilities: those formed with lse = +infinity are 0
    float lse = there ? P.lse[stat] * 1.44269504088896340736f : INFINITY;
    lse = lse == -INFINITY ? INFINITY : lse - mrf_attn_shift<T>();

    const int t0 = s.from(r0) / KT, t1 = r0 <= i1 ? (s.to(i1) + KT - 1) / KT : 0;
    const T *k = (const T *)P.k + b * P.ks[0] + hk * P.ks[2], *v = (const T *)P.v + b * P.vs[0] + hk * P.vs[2];
    Rows kr, vr;
    typename decltype(line)::Next bias_next = {};
    const auto load = [&](int t) __attribute__((always_inline)) {
        kr.load(k + (long long)t * KT * P.ks[1], P.ks[1], s.nk - t * KT, P.D);
        vr.load(v + (long long)t * KT * P.vs[1], P.vs[1], s.nk - t * KT, P.D);
        if constexpr (BIAS) line.fetch(P, s, h, (long long)(t + 1) * KT - r0 - (ROWS - 1), bias_next);
    };
    const auto store = [&](int buf) __attribute__((always_inline)) {
        kr.store(lds[buf][0]);
        vr.store(lds[buf][1]);
        if constexpr (BIAS) line.put(buf, bias_next);
    };
    constexpr bool MEAN = sizeof(T) == 2;
    typename MrfSum<T>::type dq[DP / 32];      // sums of dS k, and of P k
    mrf_acc mean[MEAN ? DP / 32 : 1];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) dq[d][e] = 0.0f, mean[MEAN ? d : 0][e] = 0.0f;
    MrfRange<T> range;
    float left = 0.0f, lost = 0.0f;      // sum of dS, a block of 32 keys at a time: it rises and falls again, and what is left shall be no roundings of its way

    if (t0 < t1) {
        if constexpr (BIAS) line.ahead(P, s, (long long)t0 * KT - r0 - (ROWS - 1), bias_next);
        load(t0);
        store(0);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1, k0 = t * KT;
        if (t + 1 < t1) load(t + 1);
        if (w0 <= w1 && k0 < s.to(w1) && k0 + KT > s.from(w0)) {
            const bool whole = k0 >= w1 + s.lo && k0 + KT - 1 <= w0 + s.hi && k0 + KT <= s.nk;
            const int from = i + s.lo - k0, to = min(i + s.hi + 1, s.nk) - k0;
            const bool flat = !BIAS || line.flat(buf);
            const float times = flat ? P.c : 1.0f, less = BIAS && flat ? lse - line.value[buf][0] : lse;
#pragma unroll 1
            for (int u = 0; u < U; ++u) {
                const T *const at = lds[0][0] + 32 * u * Rows::LD;
                mrf_acc c, dp;
#pragma unroll
                for (int e = 0; e < 16; ++e) c[e] = dp[e] = 0.0f;
                mrf_ahead<STEPS, mrf_attn_group<T, DP>()>([&](int n) { return MrfTwo<frag>{places.along(at, n), places.along(at + TILE, n)}; },
                                                          [&](int n, const MrfTwo<frag> &f) {
                                                              c = mrf_mma(f.a, qf[n], c);
                                                              dp = mrf_mma(f.b, gf[n], dp);
                                                          });
                if (BIAS && !flat) {
                    mrf_stay_branch();
                    const float *const values = line.value[buf] + ROWS - 1 - (wv * 32 + (lane & 31)) + 32 * u;
#pragma unroll
                    for (int e = 0; e < 16; ++e) c[e] = fmaf(c[e], P.c, values[mrf_acc_row(e, half)]);
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) c[e] = __builtin_amdgcn_exp2f(fmaf(c[e], times, -less));
                if (!whole) {
                    mrf_stay_branch();
                    const unsigned rows_in = mrf_rows_between(from - 32 * u, to - 32 * u, half);
#pragma unroll
                    for (int e = 0; e < 16; ++e) c[e] = mrf_keep(mrf_row_bits(rows_in, e), c[e]);
                }
                float of_block = 0.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    dp[e] = c[e] * (dp[e] - delta);
                    of_block += dp[e];
                }
                mrf_add(left, lost, of_block);
                range.fit(dp, dq);
                const frag sf[2] = {mrf_acc_frag<T>(dp, 0), mrf_acc_frag<T>(dp, 1)}, pf[2] = {mrf_acc_frag<T>(c, 0), mrf_acc_frag<T>(c, 1)};
                if constexpr (MEAN)
                    mrf_ahead<STEPS, mrf_attn_group<T, DP>()>([&](int n) { return places.across(at + 16 * (n / (DP / 32)) * Rows::LD, n % (DP / 32)); },
                                                              [&](int n, const frag &f) {
                                                                  const int x = n / (DP / 32), d = n % (DP / 32);
                                                                  dq[d] = mrf_mma(f, sf[x], dq[d]);
                                                                  mean[d] = mrf_mma(f, pf[x], mean[d]);
                                                              });
                else
                    mrf_add_block<DP>(places, at, Rows::LD, sf, dq);
            }
        }
        if (t + 1 < t1) store(buf ^ 1);
        places.move(buf ? -2 * TILE : 2 * TILE);
        __syncthreads();
    }
    left = mrf_halves_sum(left) * mrf_attn_unshift<T>();
    if (i >= P.Q) return;
    if (half == 0) P.delta[stat] = delta + left;
    if (!P.dq) return;
    T *const out = (T *)P.dq + row;
    const float undo = range.undo(), scale = P.scale * mrf_attn_unshift<T>();
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            float x[4];
#pragma unroll
            for (int n = 0; n < 4; ++n) x[n] = (MEAN ? fmaf(-left, mean[MEAN ? d : 0][e + n], (float)dq[d][e + n] * undo) : (float)dq[d][e + n]) * scale;
            mrf_store4(out, 32 * d + mrf_acc_row(e, half), P.D, x);
        }
}

// Query tiles that a workgroup of keys k0 .. goes through: those with a query that may see one of its keys
template <int QT> __device__ inline void mrf_attn_query_tiles(const MrfAttnBatch &s, int k0, int &t0, int &t1)
{
    const int k1 = min(k0 + 128, s.nk) - 1;
    const long long from = max((long long)k0 - s.hi, 0LL), to = min((long long)k1 - s.lo + 1, (long long)s.nq);
    t0 = k0 <= k1 && from < to ? (int)(from / QT) : 0;
    t1 = k0 <= k1 && from < to ? (int)((to + QT - 1) / QT) : 0;
}

// ---- dk, dv, sums of dS along diagonals
//
// TABLE: dS of 32 queries x 32 keys is put into LDS with each query's row moved by one against the next, so that a column holds a diagonal (places that none
// falls on stay 0), and a lane sums a column.  A wavefront has 32 keys and goes through the queries upwards: of the 63 diagonals of a
// block (of the last lane there is none) the later 31 go on in the next one, whose lanes are 32 less, and 32 are done and written.  An entry of the line: query - (key - first key) + 31, less the
// first query of the strip's tiles.
// 63 entries a row, and 32 that are left free each time after rows 3, 11, 19 and 27: so the halves of a wavefront, four rows apart, fall on the two halves of the banks.
__host__ __device__ constexpr int mrf_skew(int row) { return 63 * row + 32 * ((row + 4) / 8); }
constexpr int MRF_SKEWED = mrf_skew(31) + 63;

// Wavefronts of a SIMD.  Heads of up to 32 entries wait for the look-ups and for LDS more than for products: 192 sequences of 624 keys, 4 heads of 32 in a
// band of 97, take 146 us with three and 177 with two.  Heads of 64 have no room for three (nor has the queries' kernel: 482 us then instead of 194 for 4 sequences
// of 2,048, 16 heads of 64; for heads of 32 three are as fast as two).
// The keys' kernel for heads of 32 with the table's gradient keeps 60 bytes a lane in scratch memory for it (and has no accumulation registers, beside which that would not do).
// Heads of 128 have room for two where dv is a launch of its own: 2 sequences of 4,160, 4 heads on one of 128, 208 us instead of 380.
//
// DK, DV: which of the two it sums.  Both, where their sums and the keys and values fit into the registers, else one launch for each.
template <class T, int DP, bool BIAS, bool TABLE, bool DK, bool DV>
__global__ void __launch_bounds__(256, (sizeof(T) == 4 || (DP == 128 && DK) ? 1 : DP >= 64 ? 2 : 3)) mrf_attn_bwd_keys(const MrfAttnParams P)
{
    constexpr int QT = mrf_attn_bwd_rows<T>(), NT = 256, KEYS = 128, LINE = KEYS + QT;
    typedef MrfRows<T, DP, QT, NT> Rows;
    typedef typename MrfFrag<T>::type frag;
    constexpr int TILE = QT * Rows::LD, U = QT / 32, STEPS = DP / 16;
    __shared__ __align__(16) T lds[2][2][TILE];      // queries, gradients of the outputs
    __shared__ __align__(16) float ldsL[2][QT], ldsD[2][QT];
    __shared__ MrfLine<BIAS ? LINE : 1> line;
    __shared__ float skew[TABLE ? 4 : 1][TABLE ? MRF_SKEWED : 1];
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5;
    // (the keys that most queries see first; part blockIdx.y of the heads that share them)
    const int bh = blockIdx.x % (P.B * P.Hk), block = (int)(blockIdx.x / (P.B * P.Hk)), group = P.G / P.shares;
    const int b = bh / P.Hk, hk = bh % P.Hk;
    const MrfAttnBatch s(P, b);
    MrfPlaces<T, DP, Rows::LD> places;
    places.template init<Rows>();
    const int k0 = block * KEYS, j = k0 + wv * 32 + (lane & 31), w0 = k0 + wv * 32, w1 = min(w0 + 31, s.nk - 1);
    int t0, t1;
    mrf_attn_query_tiles<QT>(s, k0, t0, t1);

    frag kf[DP / 16] = {}, vf[DK ? DP / 16 : 1] = {};
    if (w0 <= w1) {
        const int at = min(j, w1);
        const T *k = (const T *)P.k + b * P.ks[0] + at * P.ks[1] + hk * P.ks[2], *v = (const T *)P.v + b * P.vs[0] + at * P.vs[1] + hk * P.vs[2];
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) {
            kf[t] = mrf_load8(k, 16 * t + 8 * half, P.D, j < s.nk);
            if constexpr (DK) vf[t] = mrf_load8(v, 16 * t + 8 * half, P.D, j < s.nk);
        }
    }
    if constexpr (TABLE)
        for (int n = lane; n < MRF_SKEWED; n += 64) skew[wv][n] = 0.0f;
    typename MrfSum<T>::type dk[DK ? DP / 32 : 1], dv[DV ? DP / 32 : 1];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) dk[DK ? d : 0][e] = 0.0f, dv[DV ? d : 0][e] = 0.0f;

    MrfRange<T> range;
    Rows qr, gr;
    float lse_next = 0.0f, delta_next = 0.0f;
    typename decltype(line)::Next bias_next = {};
    int now = 0;      // which of the two tiles `places` are in
    for (int g = 0; g < group; ++g) {
        const int h = hk * P.G + blockIdx.y * group + g;
        const T *q = (const T *)P.q + b * P.qs[0] + h * P.qs[2], *go = (const T *)P.dout + ((long long)b * P.Q * P.Hq + h) * P.D;
        const long long stat = ((long long)b * P.Hq + h) * P.Q;
        const auto load = [&](int t) __attribute__((always_inline)) {
            qr.load(q + (long long)t * QT * P.qs[1], P.qs[1], s.nq - t * QT, P.D);
            gr.load(go + (long long)t * QT * P.Hq * P.D, (long long)P.Hq * P.D, s.nq - t * QT, P.D);
            if ((int)threadIdx.x < QT) {
                const int i = t * QT + (int)threadIdx.x;
                lse_next = i < s.nq ? P.lse[stat + i] * 1.44269504088896340736f : INFINITY;
                lse_next = lse_next == -INFINITY ? INFINITY : lse_next - mrf_attn_shift<T>();
                delta_next = i < s.nq ? P.delta[stat + i] : 0.0f;
            }
            if constexpr (BIAS) line.fetch(P, s, h, (long long)k0 - (long long)(t + 1) * QT - (QT - 1), bias_next);
        };
        const auto store = [&](int buf) __attribute__((always_inline)) {
            qr.store(lds[buf][0]);
            gr.store(lds[buf][1]);
            if ((int)threadIdx.x < QT) {
                ldsL[buf][threadIdx.x] = lse_next;
                ldsD[buf][threadIdx.x] = delta_next;
            }
            if constexpr (BIAS) line.put(buf, bias_next);
        };
        float *const to_line = TABLE ? P.lines + (((size_t)b * P.Hq + h) * P.strips + block * 4 + wv) * P.line : nullptr;
        float goes_on = 0.0f;
        if (t0 < t1) {
            if constexpr (BIAS) line.ahead(P, s, (long long)k0 - (long long)t0 * QT - (QT - 1), bias_next);
            load(t0);
            store(now);
        }
        __syncthreads();
        for (int t = t0; t < t1; ++t) {
            const int buf = now, q0 = t * QT;
            if (t + 1 < t1) load(t + 1);
            const int q1 = min(q0 + QT, s.nq) - 1;
            const bool any = w0 <= w1 && q1 + s.hi >= w0 && q0 + s.lo <= w1;
            const bool whole = any && w0 >= q1 + s.lo && w0 + 31 <= q0 + s.hi && q0 + QT <= s.nq && w0 + 32 <= s.nk;
            // queries that may see this lane's key: [from, to) of the tile
            const int from = j - s.hi - q0, to = j < s.nk ? min(j - s.lo + 1, s.nq) - q0 : 0;
            const bool flat = !BIAS || line.flat(buf);
            const float times = flat ? P.c : 1.0f, level = BIAS && flat ? line.value[buf][0] : 0.0f;
            // (heads of 128: 432 us and 420 for 4 sequences of 2,048, 16 heads; the queries' kernel, which has more to keep, 343 and 416)
            constexpr int TOGETHER = sizeof(T) == 2 && DP == 128 && DK && DV ? 2 : 1;
#pragma unroll TOGETHER
            for (int u = 0; u < U; ++u) {
                float sum = goes_on;
                if (any) {
                    const T *const at = lds[0][0] + 32 * u * Rows::LD;
                    mrf_acc c, dp;
#pragma unroll
                    for (int e = 0; e < 16; ++e) c[e] = dp[e] = 0.0f;
                    mrf_ahead<STEPS, mrf_attn_group<T, DP>()>(
                        [&](int n) {
                            MrfTwo<frag> f = {places.along(at, n), {}};
                            if constexpr (DK) f.b = places.along(at + TILE, n);
                            return f;
                        },
                        [&](int n, const MrfTwo<frag> &f) {
                            c = mrf_mma(f.a, kf[n], c);
                            if constexpr (DK) dp = mrf_mma(f.b, vf[DK ? n : 0], dp);
                        });
                    if (BIAS && !flat) {
                        mrf_stay_branch();
                        const float *const values = line.value[buf] + QT - 1 + (wv * 32 + (lane & 31)) - 32 * u;
#pragma unroll
                        for (int e = 0; e < 16; ++e) c[e] = fmaf(c[e], P.c, values[-mrf_acc_row(e, half)]);
                    }
#pragma unroll
                    for (int e4 = 0; e4 < 16; e4 += 4) {
                        const int r4 = 32 * u + mrf_acc_row(e4, half);
                        const float4 L = *(const float4 *)&ldsL[buf][r4], D = *(const float4 *)&ldsD[buf][r4];
                        const float lse[4] = {L.x, L.y, L.z, L.w}, delta[4] = {D.x, D.y, D.z, D.w};
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            c[e4 + n] = __builtin_amdgcn_exp2f(fmaf(c[e4 + n], times, BIAS ? level - lse[n] : -lse[n]));
                            dp[e4 + n] -= delta[n];
                        }
                    }
                    if (!whole) {
                        mrf_stay_branch();
                        const unsigned rows_in = mrf_rows_between(from - 32 * u, to - 32 * u, half);
#pragma unroll
                        for (int e = 0; e < 16; ++e) c[e] = mrf_keep(mrf_row_bits(rows_in, e), c[e]);
                    }
#pragma unroll
                    for (int e = 0; e < 16; ++e) dp[e] *= c[e];
                    if constexpr (TABLE) {
                        // Where all offsets of the tile have a bucket, and all its pairs count, it does not matter on which of its diagonals they are.
                        if (flat && whole) {
                            float mine = 0.0f;
#pragma unroll
                            for (int e = 0; e < 16; ++e) mine += dp[e];
                            mine = mrf_halves_sum(mine);
                            sum += half == 0 ? mine : 0.0f;
                        } else {
                            mrf_stay_branch();
                            float *const skewed = skew[TABLE ? wv : 0];
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const int r = mrf_acc_row(e, half);
                                skewed[mrf_skew(r) + r - (lane & 31) + 31] = dp[e];
                            }
                            mrf_wave_lds_fence();
                            float part[4] = {};
#pragma unroll
                            for (int r = 0; r < 32; ++r) part[r % 4] += skewed[mrf_skew(r) + min(lane, 62)];
                            sum += lane < 63 ? (part[0] + part[1]) + (part[2] + part[3]) : 0.0f;
                            mrf_wave_lds_fence();
                        }
                    }
                    frag pf[2], sf[2];
                    if constexpr (DK) {
                        range.fit(dp, dk);
                        sf[0] = mrf_acc_frag<T>(dp, 0), sf[1] = mrf_acc_frag<T>(dp, 1);
                    }
                    if constexpr (DV) pf[0] = mrf_acc_frag<T>(c, 0), pf[1] = mrf_acc_frag<T>(c, 1);
                    if constexpr (sizeof(T) == 4) {
                        if constexpr (DV) mrf_add_block<DP>(places, at + TILE, Rows::LD, pf, dv);
                        if constexpr (DK) mrf_add_block<DP>(places, at, Rows::LD, sf, dk);
                    } else {
                        mrf_ahead<STEPS, mrf_attn_group<T, DP>()>(
                            [&](int n) {
                                const T *const row = at + 16 * (n / (DP / 32)) * Rows::LD;
                                MrfTwo<frag> f = {};
                                if constexpr (DV) f.a = places.across(row + TILE, n % (DP / 32));
                                if constexpr (DK) f.b = places.across(row, n % (DP / 32));
                                return f;
                            },
                            [&](int n, const MrfTwo<frag> &f) {
                                const int x = n / (DP / 32), d = n % (DP / 32);
                                if constexpr (DV) dv[DV ? d : 0] = mrf_mma(f.a, pf[x], dv[DV ? d : 0]);
                                if constexpr (DK) dk[DK ? d : 0] = mrf_mma(f.b, sf[x], dk[DK ? d : 0]);
                            });
                    }
                }
                if constexpr (TABLE) {
                    if (half == 0) to_line[(t - t0) * QT + 32 * u + lane] = sum * mrf_attn_unshift<T>();
                    goes_on = __shfl(sum, lane | 32);
                    if (half) goes_on = 0.0f;
                }
            }
            if (t + 1 < t1) {
                store(buf ^ 1);
                now ^= 1;
                places.move(now ? 2 * TILE : -2 * TILE);
            }
            __syncthreads();
        }
        if constexpr (TABLE)
            if (half == 0 && t0 < t1) to_line[(t1 - t0) * QT + lane] = goes_on * mrf_attn_unshift<T>();
    }
    if (j >= P.K) return;
    const long long row = (((long long)b * P.K + j) * P.Hk + hk) * P.D, all = (long long)P.B * P.K * P.Hk * P.D;
    const float ks = P.scale * mrf_attn_unshift<T>() * range.undo(), vs = mrf_attn_unshift<T>();
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            float x[4];
            const int at = 32 * d + mrf_acc_row(e, half);
            if constexpr (DK) {
#pragma unroll
                for (int n = 0; n < 4; ++n) x[n] = (float)dk[DK ? d : 0][e + n] * ks;
                if (P.shares > 1) mrf_store4(P.share + 2 * blockIdx.y * all + row, at, P.D, x);
                else if (P.dk) mrf_store4((T *)P.dk + row, at, P.D, x);
            }
            if constexpr (DV) {
#pragma unroll
                for (int n = 0; n < 4; ++n) x[n] = (float)dv[DV ? d : 0][e + n] * vs;
                if (P.shares > 1) mrf_store4(P.share + (2 * blockIdx.y + 1) * all + row, at, P.D, x);
                else if (P.dv) mrf_store4((T *)P.dv + row, at, P.D, x);
            }
        }
}

// Sums of the parts that several workgroups (512 at most) made of a head of keys, in their order, in 64 bits: dk, dv
template <class T> __global__ void __launch_bounds__(256) mrf_attn_shares(const MrfAttnParams P)
{
    typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
    const long long all = (long long)P.B * P.K * P.Hk * P.D, at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= all) return;
    T *const out = (T *)(blockIdx.y ? P.dv : P.dk);
    const int left = all - at < 4 ? (int)(all - at) : 4;
    double x[4] = {};
    for (int s = 0; s < P.shares; ++s) {
        const float *const p = P.share + (2 * s + blockIdx.y) * all + at;
        if (left == 4) {
            const vec v = *(const vec *)p;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] += v[j];
        } else {
            for (int j = 0; j < left; ++j) x[j] += p[j];
        }
    }
    const float sums[4] = {(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
    if (out) mrf_store4(out + at, 0, left, sums);
}

// Gradient of the table: what the lines hold of a diagonal, summed over the strips of keys that it crosses, belongs to the bucket of its offset.  A workgroup
// goes through `pieces` pieces of 256 offsets of a sequence, a thread its offset's strips, which it adds in 64 bits as long as the bucket stays the same (512 strips that
// are all alike, each rounded the same way, left sums of 32 bits off by 1e-5); each thread has a sum of its own for each of MRF_TABLE_BUCKETS buckets in LDS, which meet at the end
// in a fixed tree.  More buckets: a layer of workgroups for each MRF_TABLE_BUCKETS of them.
constexpr int MRF_TABLE_BUCKETS = 32;

template <int QT> __global__ void __launch_bounds__(256) mrf_attn_buckets(const MrfAttnParams P)
{
    __shared__ float sums[MRF_TABLE_BUCKETS][256];
    const int tid = threadIdx.x, part = blockIdx.x, h = blockIdx.y, first_bucket = blockIdx.z * MRF_TABLE_BUCKETS;
    const long long n = (long long)P.Q + P.K - 1, blocks = (n + 255) / 256, all = blocks * P.B;
    const long long x0 = part * P.pieces, x1 = x0 + P.pieces < all ? x0 + P.pieces : all;
#pragma unroll
    for (int k = 0; k < MRF_TABLE_BUCKETS; ++k) sums[k][tid] = 0.0f;
    int bucket = 0;
    double sum = 0.0;      // of `bucket`
    for (long long x = x0; x < x1; ++x) {
        const int b = (int)(x / blocks);
        const long long at = (x - b * blocks) * 256 + tid;
        const MrfAttnBatch s(P, b);
        const long long offset = at - (P.Q - 1);
        if (at >= n || offset < s.lo || offset > s.hi) continue;
        long long m = s.map + offset;
        m = m < 0 ? 0 : m >= P.n_offsets ? P.n_offsets - 1 : m;
        int k = P.bucket_of[m];
        k = (k < 0 ? 0 : k >= P.n_buckets ? P.n_buckets - 1 : k) - first_bucket;
        if (k < 0 || k >= MRF_TABLE_BUCKETS) continue;
        // strips whose keys have a query at that offset: key - offset in [0, nq)
        const float *const lines = P.lines + ((size_t)b * P.Hq + h) * P.strips * P.line;
        const int first = (int)(max(offset, 0LL) / 128 * 4), last = (int)min(offset + s.nq - 1, (long long)s.nk - 1);
        if (k != bucket) {
            sums[bucket][tid] += (float)sum;
            bucket = k;
            sum = 0.0;
        }
        // (a workgroup's four strips have the same tiles; the loads of two workgroups' are on their way together)
        for (int strip = first; strip <= last / 32 && last >= 0; strip += 8) {
            float v[8];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                int t0, t1;
                mrf_attn_query_tiles<QT>(s, 32 * (strip + 4 * y), t0, t1);
                const int entry = (int)(32 * (strip + 4 * y) - offset + 31);
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int e = entry + 32 * w;
                    const bool in = t0 < t1 && e >= t0 * QT && e < t1 * QT + 32;
                    const float value = lines[in ? (strip + 4 * y + w) * (long long)P.line + e - t0 * QT : 0];
                    v[4 * y + w] = in ? value : 0.0f;
                }
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) sum += (v[4 * y] + v[4 * y + 1]) + (v[4 * y + 2] + v[4 * y + 3]);
        }
    }
    sums[bucket][tid] += (float)sum;
    for (int w = 128; w > 0; w /= 2) {
        __syncthreads();
        for (int y = tid; y < MRF_TABLE_BUCKETS * w; y += 256) sums[y / w][y % w] += sums[y / w][y % w + w];
    }
    __syncthreads();
    if (tid < MRF_TABLE_BUCKETS && first_bucket + tid < P.n_buckets)
        P.partial[((size_t)h * P.n_buckets + first_bucket + tid) * P.parts + part] = sums[tid][0];
}

// A wavefront sums the parts of a bucket (none: 0), and goes on to another where there are more than a grid has wavefronts.
constexpr long long MRF_TABLE_GROUPS = 1 << 22;
static __global__ void __launch_bounds__(256) mrf_attn_table(const MrfAttnParams P)
{
    const int lane = threadIdx.x & 63;
    for (long long x = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); x < (long long)P.Hq * P.n_buckets; x += gridDim.x * 4LL) {
        const int h = (int)(x / P.n_buckets), k = (int)(x - (long long)h * P.n_buckets);
        float sum = 0.0f;
        for (int p = lane; p < P.parts; p += 64) sum += P.partial[x * P.parts + p];
        sum = mrf_lanes_sum<64>(sum);
        if (lane == 0) P.dtable[P.heads_last ? (size_t)k * P.Hq + h : (size_t)h * P.n_buckets + k] = sum;
    }
}

namespace mrf_host {

template <class T, int DP> static int attention_back(const MrfAttnParams &P, hipStream_t st)
{
    const bool pairs = P.B && P.Q && P.K;
    if (P.B && P.Q) {
        const unsigned grid = (unsigned)((long long)P.B * P.Hq * ((P.Q + 127) / 128));
        if (P.table) mrf_attn_bwd_queries<T, DP, true><<<grid, 256, 0, st>>>(P);
        else mrf_attn_bwd_queries<T, DP, false><<<grid, 256, 0, st>>>(P);
    }
    if (P.B && P.K && (P.dk || P.dv || P.dtable)) {
        const dim3 grid((unsigned)((long long)P.B * P.Hk * ((P.K + 127) / 128)), (unsigned)P.shares);
        constexpr bool ONE = DP == 128 && sizeof(T) == 4;      // one of the two at a time
        if (P.dtable && pairs) mrf_attn_bwd_keys<T, DP, true, true, true, DP != 128><<<grid, 256, 0, st>>>(P);
        else if (P.table) mrf_attn_bwd_keys<T, DP, true, false, true, !ONE><<<grid, 256, 0, st>>>(P);
        else mrf_attn_bwd_keys<T, DP, false, false, true, !ONE><<<grid, 256, 0, st>>>(P);
        if constexpr (DP == 128)
            if (P.dv && (ONE || (P.dtable && pairs))) {
                if (P.table) mrf_attn_bwd_keys<T, DP, true, false, false, true><<<grid, 256, 0, st>>>(P);
                else mrf_attn_bwd_keys<T, DP, false, false, false, true><<<grid, 256, 0, st>>>(P);
            }
        if (P.shares > 1 && (P.dk || P.dv)) {
            const long long n = ((long long)P.B * P.K * P.Hk * P.D + 1023) / 1024;
            mrf_attn_shares<T><<<dim3((unsigned)n, 2), 256, 0, st>>>(P);
        }
    }
    if (P.dtable) {
        if (pairs) {
            const dim3 grid((unsigned)P.parts, (unsigned)P.Hq, (unsigned)((P.n_buckets + MRF_TABLE_BUCKETS - 1) / MRF_TABLE_BUCKETS));
            mrf_attn_buckets<mrf_attn_bwd_rows<T>()><<<grid, 256, 0, st>>>(P);
        }
        const long long groups = ((long long)P.Hq * P.n_buckets + 3) / 4;
        mrf_attn_table<<<(unsigned)(groups < MRF_TABLE_GROUPS ? groups : MRF_TABLE_GROUPS), 256, 0, st>>>(P);
    }
    return launch_status("mrf_attn_bwd");
}

template <class T> [[maybe_unused]] static int attention_back_typed(const MrfAttnParams &P, hipStream_t st)
{
    if (P.D <= 32) return attention_back<T, 32>(P, st);
    if (P.D <= 64) return attention_back<T, 64>(P, st);
    if constexpr (sizeof(T) == 4) return attention_back<T, 128>(P, st);
    else return attention_backward_128(P, std::is_same<T, mrf_f16>::value ? MRF_F16 : MRF_BF16, st);
}

#if defined(MRF_ATTENTION_F32)
int attention_backward_f32(const MrfAttnParams &P, hipStream_t st) { return attention_back_typed<float>(P, st); }
}  // namespace mrf_host
#elif defined(MRF_ATTENTION_128)
int attention_backward_128(const MrfAttnParams &P, int type, hipStream_t st)
{
    return type == MRF_F16 ? attention_back<mrf_f16, 128>(P, st) : attention_back<mrf_bf16, 128>(P, st);
}
}  // namespace mrf_host
#else

static size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// A line for every strip of 32 keys: an entry for each query, as far as whole tiles reach, and 32 more.  The tiles are those that the 128 keys around the strip may be seen from:
// where the band has two ends, 128 queries and its width, in tiles that these begin and end anywhere in.
static void attention_lines(MrfAttnParams &P)
{
    const long long queries = ((long long)P.Q + 63) / 64 * 64, seen = P.last - P.first + 128, band = seen < 0 ? 0 : (seen + 126) / 64 * 64;
    P.strips = (int)(((long long)P.K + 127) / 128 * 4);
    P.line = (int)(band < queries ? band : queries) + 32;
}

// Workgroups of a head that sum the table's gradient, and pieces of 256 offsets that each goes through: workgroups for the whole card four times over, as far as there are
// pieces for them (16 heads of 2,048 queries and keys in 4 batches: 22 us with half of that and the strips of one workgroup at a time, 15 now)
static void attention_parts(MrfAttnParams &P)
{
    const long long all = P.Q && P.K ? ((long long)P.Q + P.K - 1 + 255) / 256 * P.B : 0;
    long long parts = 1024 / P.Hq < 1 ? 1 : 1024 / P.Hq > 256 ? 256 : 1024 / P.Hq;
    if (parts > all) parts = all;
    P.pieces = parts ? (all + parts - 1) / parts : 0;
    P.parts = parts ? (int)((all + P.pieces - 1) / P.pieces) : 0;
}

// Workgroups that share the heads of queries on a head of keys: as many as it takes for two on a compute unit, since some have far more queries to go through
// than others where those see only keys before them.
static int attention_shares(const MrfAttnParams &P)
{
    const long long grid = (long long)P.B * P.Hk * ((P.K + 127) / 128);
    int shares = 1;
    for (int n = 2; n <= P.G && grid * shares < 512; ++n)
        if (P.G % n == 0) shares = n;
    return shares;
}

static size_t attention_share_bytes(const MrfAttnParams &P, int shares)
{
    return shares > 1 ? round256(2 * (size_t)shares * P.B * P.K * P.Hk * P.D * sizeof(float)) : 0;
}

size_t attention_backward_bytes(const MrfAttnParams &given, bool table_gradient)
{
    MrfAttnParams P = given;
    size_t n = round256((size_t)P.B * P.Hq * P.Q * sizeof(float)) + attention_share_bytes(P, attention_shares(P));
    if (P.table && table_gradient && P.B && P.Q && P.K) {
        attention_lines(P);
        attention_parts(P);
        n += round256((size_t)P.B * P.Hq * P.strips * P.line * sizeof(float)) + (size_t)P.Hq * P.n_buckets * P.parts * sizeof(float);
    }
    return n ? n : 256;
}

}  // namespace mrf_host

using namespace mrf_host;

extern "C" {

int mrf_attention_backward(const mrf_attention *att, const void *grad_out, const void *out, const float *lse, void *grad_q, void *grad_k, void *grad_v,
                           float *grad_table, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    MrfAttnParams P = {};
    const int rc = attention_check(att, P);
    if (rc != MRF_OK) return rc;
    if (grad_table && !P.table) return MRF_ERR_NULL_POINTER;
    if (P.B && P.Q && (!P.q || !grad_out || !out || !lse)) return MRF_ERR_NULL_POINTER;
    if (P.B && P.K && (!P.k || !P.v)) return MRF_ERR_NULL_POINTER;
    if (!workspace) return MRF_ERR_NULL_POINTER;
    if (workspace_bytes < attention_backward_bytes(P, grad_table != nullptr)) return MRF_ERR_WORKSPACE_TOO_SMALL;
    P.dout = grad_out; P.out = (void *)out; P.lse = (float *)lse; P.dq = grad_q; P.dk = grad_k; P.dv = grad_v; P.dtable = grad_table;
    attention_lines(P);
    attention_parts(P);
    P.delta = (float *)workspace;
    P.shares = attention_shares(P);
    P.share = (float *)((char *)workspace + round256((size_t)P.B * P.Hq * P.Q * sizeof(float)));
    P.lines = (float *)((char *)P.share + attention_share_bytes(P, P.shares));
    P.partial = (float *)((char *)P.lines + round256((size_t)P.B * P.Hq * P.strips * P.line * sizeof(float)));
    hipStream_t st = (hipStream_t)hip_stream;
    if (att->type == MRF_F32) return attention_backward_f32(P, st);
    return att->type == MRF_F16 ? attention_back_typed<mrf_f16>(P, st) : attention_back_typed<mrf_bf16>(P, st);
}

}  // extern "C"
#endif
