// Attention of heads with a bias by bucketed distance, forward (see mrf_attention_forward in the header for the formulas).
//
// A wavefront has 32 queries of a head (or of few queries those of all the heads that share keys), its workgroup goes through the keys that they may
// see, tile after tile, in one pass: maximum and sum of the exponentials of a query run along, and what was summed is scaled where the
// maximum rises.  Scores are formed as keys x queries, so that a lane has a single query: its maximum and sum are within two lanes, and its
// probabilities are an operand of the second product as they are.
//
// What bounds it: with 128 entries the matrix units, fed from LDS at the rate they multiply at; with 32 the exponential and the six operations around it, which take
// longer than the products; in 32 bits the matrix units; in bands, with look-ups of a bias and with few tiles a workgroup the waiting (40 to 60 % of the wavefronts' cycles).  4
// sequences of 2,048, 16 heads, without a mask: heads of 32 in 70 us (490 TFLOP/s), 64 105 (650), 128 154 (890; a
// plain product of 8,192^3 reaches 1,082); 64 in 32 bits 607 (113; 153).  A single query of 16 heads on each of 16 caches of up to 16,411 keys, 4 heads of 128: 75 us, 4.4
// TB/s, and 5 to join the parts (a copy reaches 5.1).
#include "mrfmp_attention.h"

#include <type_traits>

// Keys of a tile: as many as two tiles of keys and values in LDS leave two workgroups (32 bits: one or two) on a compute unit.
template <class T, int NW> constexpr int mrf_attn_keys() { return sizeof(T) == 4 || NW == 1 ? 32 : 64; }

// What was summed is scaled only where a maximum rises by more than this (in powers of two): most tiles bring one of 32 queries a new maximum.  Probabilities are then up to
// 2^8, which takes that much off what they are scaled up by in MRF_F16.
constexpr float MRF_ATTN_RISE = 8.0f;
template <class T> constexpr float mrf_attn_shift_forward() { return mrf_attn_shift<T>() > 0.0f ? mrf_attn_shift<T>() - MRF_ATTN_RISE : 0.0f; }
template <class T> constexpr float mrf_attn_unshift_forward() { return mrf_attn_shift<T>() > 0.0f ? 0x1p-7f : 1.0f; }

// Wavefronts of a SIMD: two, where their registers fit (in 32 bits not for 128 entries); three for heads of up to 64 entries in 16 bits, which wait more than they
// multiply: 192 sequences of 624 queries, 4 heads of 32 in a band of 97, with a bias, 104 us with two, 75 with three, 89 with four; 4 sequences of up to 2,048, 16 heads
// of 64, with a bias, 117 us with two, 89 with three, all of 2,048 without a bias 113 and 105.
template <class T, int DP, int NW> constexpr int mrf_attn_waves() { return NW == 1 || (sizeof(T) == 4 && DP == 128) ? 1 : sizeof(T) == 2 && DP <= 64 ? 3 : 2; }

// Wavefronts of a workgroup for many queries: with eight, a tile of keys and values of 128 entries takes half the registers on its way to LDS, and two wavefronts
// fit on a SIMD
template <class T, int DP> constexpr int mrf_attn_wide() { return sizeof(T) == 2 && DP == 128 ? 8 : 4; }

// NW wavefronts; PACK: a row is a query of a head of the group that shares keys (row = query G + head of the group), else a query of one head;
// BIAS: with a table.
template <class T, int DP, int NW, bool PACK, bool BIAS> __global__ void __launch_bounds__(64 * NW, (mrf_attn_waves<T, DP, NW>())) mrf_attn_fwd(const MrfAttnParams P)
{
    constexpr int KT = mrf_attn_keys<T, NW>(), NT = 64 * NW, ROWS = 32 * NW, LINE = ROWS + KT;
    typedef MrfRows<T, DP, KT, NT> Rows;
    typedef typename MrfFrag<T>::type frag;
    constexpr int TILE = KT * Rows::LD;
    __shared__ __align__(16) T lds[2][2][TILE];      // keys, values
    __shared__ MrfLine<BIAS && !PACK ? LINE : 1> line;
    // few queries, of several heads: the buckets at a tile's offsets, and the values of the group's heads where there is room for them
    constexpr int LEVELS = 512;
    __shared__ int ids[2][PACK && BIAS ? NW : 1][64];
    __shared__ float levels[PACK && BIAS ? LEVELS : 1];
    MrfPlaces<T, DP, Rows::LD> places;
    places.template init<Rows>();
    const int lane = threadIdx.x & 63, wv = NW == 1 ? 0 : __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), half = lane >> 5;
    const int heads = PACK ? P.Hk : P.Hq, rows = PACK ? P.Q * P.G : P.Q, blocks = (rows + ROWS - 1) / ROWS;
    // (the longest rows of causal ones first, so that the last workgroups to start are short ones; a head's blocks a fixed number apart, on one XCD as a rule)
    const int bh = blockIdx.x % (P.B * heads), block = blocks - 1 - (int)(blockIdx.x / (P.B * heads));
    const int b = bh / heads, h0 = bh % heads, hk = PACK ? h0 : h0 / P.G;
    const MrfAttnBatch s(P, b);
    const int r0 = block * ROWS, row = r0 + wv * 32 + (lane & 31);
    const int i = PACK ? row / P.G : row, h = PACK ? hk * P.G + row % P.G : h0;
    const bool there = row < rows && i < s.nq;
    // queries of the workgroup and of the wavefront
    const int i0 = PACK ? r0 / P.G : r0, i1 = min((PACK ? (r0 + ROWS - 1) / P.G : r0 + ROWS - 1), s.nq - 1);
    const int w0 = PACK ? (r0 + wv * 32) / P.G : r0 + wv * 32, w2 = PACK ? (r0 + wv * 32 + 31) / P.G : r0 + wv * 32 + 31, w1 = min(w2, s.nq - 1);

    frag qf[DP / 16] = {};
    if (w0 <= w1) {
        const T *q = (const T *)P.q + b * P.qs[0] + min(i, w1) * P.qs[1] + h * P.qs[2];
#pragma unroll
        for (int t = 0; t < DP / 16; ++t) qf[t] = mrf_load8(q, 16 * t + 8 * half, P.D, there);
    }

    int t0 = s.from(i0) / KT, t1 = i0 <= i1 ? (s.to(i1) + KT - 1) / KT : 0;
    if (P.splits > 1 && t1 > t0) {
        const int per = (t1 - t0 + P.splits - 1) / P.splits;
        t0 += blockIdx.y * per;
        t1 = min(t1, t0 + per);
    }
    const T *k = (const T *)P.k + b * P.ks[0] + hk * P.ks[2], *v = (const T *)P.v + b * P.vs[0] + hk * P.vs[2];
    Rows kr, vr;
    typename decltype(line)::Next bias_next = {};
    const auto load = [&](int t) __attribute__((always_inline)) {
        kr.load(k + (long long)t * KT * P.ks[1], P.ks[1], s.nk - t * KT, P.D);
        vr.load(v + (long long)t * KT * P.vs[1], P.vs[1], s.nk - t * KT, P.D);
        if constexpr (BIAS && !PACK) line.fetch(P, s, h0, (long long)(t + 1) * KT - r0 - (ROWS - 1), bias_next);
        if constexpr (BIAS && PACK) bias_next.bucket = mrf_attn_bucket(P, s, (long long)t * KT - w2 + lane);
    };
    const auto store = [&](int buf) __attribute__((always_inline)) {
        kr.store(lds[buf][0]);
        vr.store(lds[buf][1]);
        if constexpr (BIAS && !PACK) line.put(buf, bias_next);
        if constexpr (BIAS && PACK) ids[buf][wv][lane] = bias_next.bucket;
    };

    typename MrfSum<T>::type o[DP / 32];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
    // Maximum so far (in units of log2), and this lane's part of the sum, which tiles' own sums are added to: keys of one probability are rounded the same way each time, and
    // 16,384 of them, one after the other, left lse off by 7e-5.  (In 64 bits instead, a row of 16,411 keys took 75 us; 66 so, and 66 as it was.)
    float m = -INFINITY, l = 0.0f, lost = 0.0f;

    const bool room = BIAS && PACK && (long long)P.G * P.n_buckets <= LEVELS;
    if constexpr (BIAS && PACK) {
        if (room)
            for (int n = lane; n < P.G * P.n_buckets; n += 64) levels[n] = mrf_attn_level(P, hk * P.G + n / P.n_buckets, n % P.n_buckets);
    }
    if (t0 < t1) {
        if constexpr (BIAS && !PACK) line.ahead(P, s, (long long)t0 * KT - r0 - (ROWS - 1), bias_next);
        load(t0);
        store(0);
    }
    __syncthreads();
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1, k0 = t * KT;
        if (t + 1 < t1) load(t + 1);
        if (w0 <= w1 && k0 < s.to(w1) && k0 + KT > s.from(w0)) {
            mrf_acc c[KT / 32];
#pragma unroll
            for (int u = 0; u < KT / 32; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) c[u][e] = 0.0f;
            constexpr int STEPS = KT / 32 * DP / 16;
            mrf_ahead<STEPS, (sizeof(T) == 4 ? 1 : DP == 128 ? 2 : STEPS < 4 ? STEPS : 4)>(
                [&](int n) { return places.along(lds[0][0] + 32 * (n / (DP / 16)) * Rows::LD, n % (DP / 16)); },
                [&](int n, const frag &f) { c[n / (DP / 16)] = mrf_mma(f, qf[n % (DP / 16)], c[n / (DP / 16)]); });
            // keys that this lane's query may see: [from, to) of the tile; all of them, for most tiles
            const bool whole = k0 >= w1 + s.lo && k0 + KT - 1 <= w0 + s.hi && k0 + KT <= s.nk && (w2 == w1 || s.nq == P.Q);
            const int from = i + s.lo - k0, to = there ? min(i + s.hi + 1, s.nk) - k0 : 0;
            // (without a bias, or with the same for all, the scores stay products, whose maximum is the scores' too, and the rest goes in with the maximum: one operation)
            float top = -INFINITY, times = P.c, plus = 0.0f;
            if constexpr (BIAS && PACK) {
                // (keys of the tile less queries of the wavefront are 63 offsets at most, from k0 - w2 on)
                const auto level = [&](int id) { return room ? levels[row % P.G * P.n_buckets + id] : mrf_attn_level(P, h, id); };
                const int id = ids[buf][wv][lane], other = __builtin_amdgcn_readfirstlane(id);
                if (!__any(id != other)) {
                    plus = level(other);
                } else {
                    mrf_stay_branch();
                    times = 1.0f;
#pragma unroll
                    for (int u = 0; u < KT / 32; ++u)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int at = 32 * u + mrf_acc_row(e, half) - i + w2;
                            c[u][e] = fmaf(c[u][e], P.c, level(ids[buf][wv][at > 63 ? 63 : at < 0 ? 0 : at]));
                        }
                }
            } else if constexpr (BIAS) {
                if (line.flat(buf)) {
                    plus = line.value[buf][0];
                } else {
                    mrf_stay_branch();
                    times = 1.0f;
                    const float *const at = line.value[buf] + ROWS - 1 - (wv * 32 + (lane & 31));
#pragma unroll
                    for (int u = 0; u < KT / 32; ++u) {
#pragma unroll
                        for (int e = 0; e < 16; ++e) c[u][e] = fmaf(c[u][e], P.c, at[32 * u + mrf_acc_row(e, half)]);
                        __builtin_amdgcn_sched_barrier(0);      // (not all values at a time: they would not fit)
                    }
                }
            }
            if (!whole) {
                mrf_stay_branch();
#pragma unroll
                for (int u = 0; u < KT / 32; ++u) {
                    const unsigned rows_in = mrf_rows_between(from - 32 * u, to - 32 * u, half);
#pragma unroll
                    for (int e = 0; e < 16; ++e) c[u][e] = mrf_keep_or_lowest(mrf_row_bits(rows_in, e), c[u][e]);
                }
            }
#pragma unroll
            for (int u = 0; u < KT / 32; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) top = fmaxf(top, c[u][e]);
            top = mrf_halves_max(top);
            top = fmaxf(m, fmaf(top, times, plus));
            const float base = top == -INFINITY ? 0.0f : top;
            if (__any(top > m + MRF_ATTN_RISE)) {
                const float less = __builtin_amdgcn_exp2f(m - base);
                l *= less;
                lost *= less;
#pragma unroll
                for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[d][e] *= less;
                m = top;
            }
            const float low = (m == -INFINITY ? 0.0f : m) - mrf_attn_shift_forward<T>() - plus;
            frag p[2];
            float of_tile = 0.0f;
            const auto probabilities = [&](int y) {
                mrf_acc &x = c[y / 2];
#pragma unroll
                for (int e = 8 * (y % 2); e < 8 * (y % 2) + 8; ++e) {
                    x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], times, -low));
                    of_tile += x[e];
                }
                p[y % 2] = mrf_acc_frag<T>(x, y % 2);
            };
            if constexpr (sizeof(T) == 4) {
                static_assert(KT == 32, "two parts");
                probabilities(0);
                probabilities(1);
                mrf_add_block<DP>(places, lds[0][1], Rows::LD, p, o);
            } else {
                // 16 keys at a time: their probabilities, and their values on the way, while those before are multiplied
                frag vf[2][DP / 32];
                const auto part = [&](int y) {
                    probabilities(y);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) vf[y % 2][d] = places.across(lds[0][1] + 16 * y * Rows::LD, d);
                };
                part(0);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int y = 0; y < KT / 16; ++y) {
                    if (y + 1 < KT / 16) part(y + 1);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) o[d] = mrf_mma(vf[y % 2][d], p[y % 2], o[d]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            mrf_add(l, lost, of_tile);
        }
        if (t + 1 < t1) store(buf ^ 1);
        places.move(buf ? -2 * TILE : 2 * TILE);
        __syncthreads();
    }

    l = mrf_halves_sum(l) * mrf_attn_unshift_forward<T>();
    if (row >= rows) return;
    if (P.splits > 1) {
        const long long n = (long long)P.B * P.Hq * P.Q, at = ((long long)b * P.Hq + h) * P.Q + i;
        float *const part = P.part + 2 * P.splits * n + (blockIdx.y * n + at) * P.D;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                float x[4];
#pragma unroll
                for (int n = 0; n < 4; ++n) x[n] = (float)o[d][e + n] * mrf_attn_unshift_forward<T>();
                mrf_store4(part, 32 * d + mrf_acc_row(e, half), P.D, x);
            }
        if (half == 0) ((float2 *)P.part)[blockIdx.y * n + at] = make_float2(m, l);
        return;
    }
    const float inv = l > 0.0f ? mrf_attn_unshift_forward<T>() / l : l;      // (no keys: 0; NaN stays)
    T *const out = (T *)P.out + (((long long)b * P.Q + i) * P.Hq + h) * P.D;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            const float x[4] = {(float)o[d][e] * inv, (float)o[d][e + 1] * inv, (float)o[d][e + 2] * inv, (float)o[d][e + 3] * inv};
            mrf_store4(out, 32 * d + mrf_acc_row(e, half), P.D, x);
        }
    if (half == 0 && P.lse) P.lse[((long long)b * P.Hq + h) * P.Q + i] = l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

// Parts of the keys, joined in their order: sums of a part count 2^(its maximum - the largest).  A workgroup has a query of a head; a wavefront every fourth part,
// a lane two entries, which it adds in 64 bits (256 parts that are all alike, each rounded the same way, left sums of 32 bits off by up to 60 units in their last place).
constexpr int MRF_ATTN_SPLITS = 1024;
template <class T> __global__ void __launch_bounds__(256) mrf_attn_join(const MrfAttnParams P)
{
    __shared__ float weight[MRF_ATTN_SPLITS];
    __shared__ float scratch[2][4];
    __shared__ double sums[4][128];
    const long long n = (long long)P.B * P.Hq * P.Q, at = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const float2 *const ends = (const float2 *)P.part;
    const float *const part = P.part + 2 * P.splits * n + at * P.D;
    float top = -INFINITY, l = 0.0f;
    for (int s = tid; s < P.splits; s += 256) top = fmaxf(top, ends[s * n + at].x);
    top = -mrf_lanes_min<64>(-top);
    if (lane == 0) scratch[0][wv] = top;
    __syncthreads();
    top = fmaxf(fmaxf(scratch[0][0], scratch[0][1]), fmaxf(scratch[0][2], scratch[0][3]));
    const float base = top == -INFINITY ? 0.0f : top;
    for (int s = tid; s < P.splits; s += 256) {
        const float2 e = ends[s * n + at];
        const float w = __builtin_amdgcn_exp2f(e.x - base);
        weight[s] = w;
        l = fmaf(e.y, w, l);
    }
    l = mrf_lanes_sum<64>(l);
    if (lane == 0) scratch[1][wv] = l;
    __syncthreads();
    l = (scratch[1][0] + scratch[1][1]) + (scratch[1][2] + scratch[1][3]);
    double x = 0.0, y = 0.0;
    const int d0 = lane < P.D ? lane : 0, d1 = lane + 64 < P.D ? lane + 64 : 0;
#pragma unroll 4
    for (int s = wv; s < P.splits; s += 4) {
        const float *const p = part + s * n * P.D;
        const double w = weight[s];
        x = fma(p[d0], w, x);
        y = fma(p[d1], w, y);
    }
    sums[wv][lane] = x;
    sums[wv][lane + 64] = y;
    __syncthreads();
    const float inv = l > 0.0f ? 1.0f / l : l;
    const long long bh = at / P.Q, i = at - bh * P.Q, b = bh / P.Hq, h = bh - b * P.Hq;
    T *const out = (T *)P.out + ((b * P.Q + i) * P.Hq + h) * P.D;
    if (tid < P.D) out[tid] = mrf_from_f32<T>((float)((sums[0][tid] + sums[1][tid]) + (sums[2][tid] + sums[3][tid])) * inv);
    if (tid == 0 && P.lse) P.lse[at] = l == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

// The same for few parts of many queries: a wavefront has a query of a head, a lane two entries.
constexpr int MRF_ATTN_FEW = 8;
template <class T> __global__ void __launch_bounds__(256) mrf_attn_join_few(const MrfAttnParams P)
{
    const long long n = (long long)P.B * P.Hq * P.Q, at = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= n) return;
    const int lane = threadIdx.x & 63, d0 = lane < P.D ? lane : 0, d1 = lane + 64 < P.D ? lane + 64 : 0;
    const float2 *const ends = (const float2 *)P.part;
    const float *const part = P.part + 2 * P.splits * n + at * P.D;
    float2 end[MRF_ATTN_FEW];
    float x[MRF_ATTN_FEW], y[MRF_ATTN_FEW], top = -INFINITY, l = 0.0f, sx = 0.0f, sy = 0.0f;
#pragma unroll
    for (int s = 0; s < MRF_ATTN_FEW; ++s) {
        const int t = s < P.splits ? s : 0;
        end[s] = ends[t * n + at];
        x[s] = part[t * n * P.D + d0];
        y[s] = part[t * n * P.D + d1];
    }
#pragma unroll
    for (int s = 0; s < MRF_ATTN_FEW; ++s) top = fmaxf(top, end[s].x);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int s = 0; s < MRF_ATTN_FEW; ++s)
        if (s < P.splits) {
            const float w = __builtin_amdgcn_exp2f(end[s].x - base);
            l = fmaf(end[s].y, w, l);
            sx = fmaf(x[s], w, sx);
            sy = fmaf(y[s], w, sy);
        }
    const float inv = l > 0.0f ? 1.0f / l : l;
    const long long bh = at / P.Q, i = at - bh * P.Q, b = bh / P.Hq, h = bh - b * P.Hq;
    T *const out = (T *)P.out + ((b * P.Q + i) * P.Hq + h) * P.D;
    if (lane < P.D) out[lane] = mrf_from_f32<T>(sx * inv);
    if (lane + 64 < P.D) out[lane + 64] = mrf_from_f32<T>(sy * inv);
    if (lane == 0 && P.lse) P.lse[at] = l == 0.0f ? -INFINITY : (base + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

namespace mrf_host {

template <class T, int DP> static int attention_go(const MrfAttnParams &P, const AttnPlan &plan, hipStream_t st)
{
    const dim3 grid(plan.grid, (unsigned)P.splits);
    if (plan.pack) {
        constexpr int NW = sizeof(T) == 4 && DP == 128 ? 2 : 1;      // (a tile on its way takes half of the registers then)
        if (P.table) mrf_attn_fwd<T, DP, NW, true, true><<<grid, 64 * NW, 0, st>>>(P);
        else mrf_attn_fwd<T, DP, NW, true, false><<<grid, 64 * NW, 0, st>>>(P);
    } else {
        constexpr int NW = mrf_attn_wide<T, DP>();
        if (P.table) mrf_attn_fwd<T, DP, NW, false, true><<<grid, 64 * NW, 0, st>>>(P);
        else mrf_attn_fwd<T, DP, NW, false, false><<<grid, 64 * NW, 0, st>>>(P);
    }
    const long long queries = (long long)P.B * P.Hq * P.Q;
    if (P.splits > MRF_ATTN_FEW) mrf_attn_join<T><<<(unsigned)queries, 256, 0, st>>>(P);
    else if (P.splits > 1) mrf_attn_join_few<T><<<(unsigned)((queries + 3) / 4), 256, 0, st>>>(P);
    return launch_status("mrf_attn_fwd");
}

template <class T> static int attention_typed(const MrfAttnParams &P, const AttnPlan &plan, hipStream_t st)
{
    if (P.D <= 32) return attention_go<T, 32>(P, plan, st);
    return P.D <= 64 ? attention_go<T, 64>(P, plan, st) : attention_go<T, 128>(P, plan, st);
}

#ifdef MRF_ATTENTION_F32
int attention_forward_f32(const MrfAttnParams &P, const AttnPlan &plan, hipStream_t st) { return attention_typed<float>(P, plan, st); }
}  // namespace mrf_host
#else

int attention_check(const mrf_attention *a, MrfAttnParams &P)
{
    if (!a) return MRF_ERR_NULL_POINTER;
    const long long most = 0x7fff0000LL;
    if (a->B < 0 || a->Q < 0 || a->K < 0 || a->Hq < 1 || a->Hk < 1 || a->Hq % a->Hk || a->D < 1 || a->D > MRF_ATTENTION_LONGEST_HEAD) return MRF_ERR_BAD_SHAPE;
    if ((long long)a->Q + a->K > most || a->Hq > 32768) return MRF_ERR_BAD_SHAPE;
    // (workgroups of 256 threads: a grid has fewer than 2^32)
    const long long groups = 0xffffff, rows = a->Q > a->K ? a->Q : a->K;
    if (a->B && a->Hq * ((rows + 127) / 128) > groups / a->B) return MRF_ERR_BAD_SHAPE;
    // (and those of many queries of heads of more than 64 entries in 16 bits, forward, 512)
    const bool wide = a->D > 64 && a->type != MRF_F32 && a->Q > (a->Hq > a->Hk ? 64 : 32);
    if (wide && a->B && a->Hq * (((long long)a->Q + 255) / 256) > groups / 2 / a->B) return MRF_ERR_BAD_SHAPE;
    if (!known_type(a->type) || !(a->scale > 0.0f) || !(a->scale * 1.44269504088896340736f < INFINITY)) return MRF_ERR_BAD_ARGUMENT;
    const long long far = 1LL << 40;
    if (a->query_offset > far || a->query_offset < -far) return MRF_ERR_BAD_ARGUMENT;
    for (int i = 0; i < 3; ++i)
        if (a->q_stride[i] < 0 || a->k_stride[i] < 0 || a->v_stride[i] < 0) return MRF_ERR_BAD_ARGUMENT;
    P.B = a->B; P.Q = a->Q; P.K = a->K; P.Hq = a->Hq; P.Hk = a->Hk; P.G = a->Hq / a->Hk; P.D = a->D;
    P.scale = a->scale; P.c = a->scale * 1.44269504088896340736f;
    P.q = a->q; P.k = a->k; P.v = a->v;
    for (int i = 0; i < 3; ++i) P.qs[i] = a->q_stride[i], P.ks[i] = a->k_stride[i], P.vs[i] = a->v_stride[i];
    // (what lies beyond 2^41 bounds nothing: no sum of these wraps around)
    const long long edge = 1LL << 41;
    P.first = a->first_offset < -edge ? -edge : a->first_offset > edge ? edge : a->first_offset;
    P.last = a->last_offset < -edge ? -edge : a->last_offset > edge ? edge : a->last_offset;
    P.offset = a->query_offset; P.offsets = a->query_offsets; P.q_lengths = a->q_lengths; P.k_lengths = a->k_lengths;
    P.table = a->table; P.bucket_of = a->bucket_of; P.map_offset = a->map_offset; P.n_offsets = a->n_offsets; P.n_buckets = a->n_buckets;
    P.heads_last = a->heads_last != 0;
    if (a->table) {
        if (a->n_buckets < 1 || a->n_buckets > 65536) return MRF_ERR_BAD_SHAPE;
        if (a->map_offset > 2 * far || a->map_offset < -2 * far || a->n_offsets < 1 || a->n_offsets > far) return MRF_ERR_BAD_ARGUMENT;
        if (!a->bucket_of) return MRF_ERR_NULL_POINTER;
    }
    return MRF_OK;
}

static AttnPlan attention_plan(const MrfAttnParams &P, int type)
{
    const long long rows = (long long)P.Q * P.G;
    const int block = type != MRF_F32 && P.D > 64 ? 256 : 128, few = type == MRF_F32 && P.D > 64 ? 64 : 32;      // (as attention_go has it)
    // Few queries: a wavefront of its own for 32 of them and the heads that share their keys, instead of a workgroup for a head.  47 sequences of 739 keys, 32 heads, us as a
    // workgroup / as wavefronts: 32 queries of 64 entries 67 / 67 (8 heads on a key head 52 / 37), of 128 151 / 126 (122 / 79), in 32 bits 687 / 389; 64 queries of 64 entries
    // 73 / 108 (55 / 63), of 128 154 / 227 (127 / 121), in 32 bits 701 / 399; 100 of 128 (144 / 195).
    const bool pack = P.Q <= 32 || (P.Q <= 64 && P.D > 64 && (type == MRF_F32 || P.G > 1));
    const long long groups = pack ? (long long)P.B * P.Hk * ((rows + few - 1) / few) : (long long)P.B * P.Hq * ((P.Q + block - 1) / block);
    // parts of the keys: for eight wavefronts of few rows on a compute unit, or a workgroup of many (two, where heads are short and keys enough to pay for joining the parts:
    // 4,096 queries and keys, 4 heads of 64, 52 us with one and 45 with two, with a bias 70 and 53; 300 queries on 3,000 keys, 16 heads, 22 and 25); of four tiles at least
    const long long tiles = ((long long)P.K + 31) / 32 / (pack ? 1 : 2);
    long long splits = groups ? (pack ? 2048 : P.D <= 64 && P.K >= 4096 ? 512 : 256) / groups : 1;
    if (splits > tiles / 4) splits = tiles / 4;
    if (splits > MRF_ATTN_SPLITS) splits = MRF_ATTN_SPLITS;
    return {pack, (int)(splits < 1 ? 1 : splits), (unsigned)groups};
}

static size_t attention_forward_bytes(const MrfAttnParams &P, int type)
{
    const AttnPlan plan = attention_plan(P, type);
    return plan.splits > 1 ? (size_t)plan.splits * P.B * P.Hq * P.Q * (P.D + 2) * sizeof(float) : 0;
}

size_t attention_backward_bytes(const MrfAttnParams &P, bool table_gradient);

}  // namespace mrf_host

using namespace mrf_host;

extern "C" {

size_t mrf_attention_workspace_bytes(const mrf_attention *att, int backward)
{
    MrfAttnParams P = {};
    if (attention_check(att, P) != MRF_OK) return 0;
    return backward ? attention_backward_bytes(P, backward != MRF_BACKWARD_KEEPS_TABLE) : attention_forward_bytes(P, att->type);
}

int mrf_attention_forward(const mrf_attention *att, void *out, float *lse, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    MrfAttnParams P = {};
    const int rc = attention_check(att, P);
    if (rc != MRF_OK || P.B == 0 || P.Q == 0) return rc;
    if (!P.q || !out || (P.K && (!P.k || !P.v))) return MRF_ERR_NULL_POINTER;
    const AttnPlan plan = attention_plan(P, att->type);
    P.out = out; P.lse = lse; P.splits = plan.splits;
    if (plan.splits > 1) {
        if (!workspace) return MRF_ERR_NULL_POINTER;
        if (workspace_bytes < attention_forward_bytes(P, att->type)) return MRF_ERR_WORKSPACE_TOO_SMALL;
        P.part = (float *)workspace;
    }
    hipStream_t st = (hipStream_t)hip_stream;
    if (att->type == MRF_F32) return attention_forward_f32(P, plan, st);
    return att->type == MRF_F16 ? attention_typed<mrf_f16>(P, plan, st) : attention_typed<mrf_bf16>(P, plan, st);
}

}  // extern "C"
#endif
