// Log-probabilities of labels under the SoftMin of the final costs, and the clipped policy loss with its gradient with
// respect to the costs (see mrf_softmin_policy in the header for the formulas).
#include "mrfmp_rows.h"

#include <type_traits>

constexpr int MRF_POLICY_BLOCKS = 4096;      // workgroups at most: partial sums of the loss
// Threads of a launch over long rows: 1,024 a compute unit.  Calls one behind the other with half of that / that / twice that: 16 bits, 2,047 rows of 3,000
// 16 / 14 / 16 us, of 8,000 27 / 24 / 26, of 12,000 33 / 36 / 39, of 32,000 94 / 64 / 69, 513 of 32,000 39 / 32 / 30, 10,000 of 16,000 254 / 142 / 142; 32 bits,
// 2,047 of 8,000 30 / 28 / 31, of 12,000 39 / 42 / 46, of 32,000 117 / 109 / 108, 10,000 of 16,000 277 / 242 / 235.
constexpr int MRF_POLICY_LONG_THREADS = 262144;
constexpr int MRF_POLICY_COUNTS = 256;       // workgroups that count the mask

struct MrfPolicyParams {
    long long N;
    int L;
    const void *cost;
    const void *labels;          // [N] of label_bytes bytes
    int label_bytes;
    const float *advantage;      // entry i / per
    unsigned per;
    const float *old_logp, *ref_logp;
    const uint8_t *mask;
    float low, high;             // bounds of the ratio
    float kl, scale;             // weight of the KL term, factor on the gradient
    const float *upstream;       // another one, in device memory (NULL: 1)
    float *loss, *logp;
    void *dcost;
    long long *counts;           // [MRF_POLICY_COUNTS] counted pixels of a workgroup's share of the mask
    double *partial;             // [blocks][2] sums of J and of k
};

__device__ inline int mrf_policy_label(const MrfPolicyParams &P, long long i)
{
    const int a = P.label_bytes == 1 ? (int)((const uint8_t *)P.labels)[i] : ((const int *)P.labels)[i];
    return a < 0 ? 0 : (a < P.L ? a : P.L - 1);
}

// exp(x) for x <= 0 by the hardware's power of two: x log2(e) is rounded once, so the result is off by 2^-24 |x| + 2^-23
// relative, 6e-6 where it is smallest (x = -87).  The instruction gives 0 below 2^-126: fine for a sum that holds a 1
__device__ inline float mrf_exp_neg(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// the same for probabilities, which may be that small: the square of exp(x / 2), twice as far off
__device__ inline float mrf_exp_small(float x)
{
    const float h = __builtin_amdgcn_exp2f(x * (0.5f * 1.44269504088896340736f));
    return h * h;
}

// exp(d) - 1: the series up to d^8 near 0 (relative error 2e-10 at 0.3), where the difference would lose its digits
__device__ inline float mrf_exp_minus_1(float d)
{
    float p = 1.0f / 40320.0f;
    p = fmaf(p, d, 1.0f / 5040.0f);
    p = fmaf(p, d, 1.0f / 720.0f);
    p = fmaf(p, d, 1.0f / 120.0f);
    p = fmaf(p, d, 1.0f / 24.0f);
    p = fmaf(p, d, 1.0f / 6.0f);
    p = fmaf(p, d, 0.5f);
    p = fmaf(p, d, 1.0f);
    return fabsf(d) < 0.3f ? p * d : __builtin_amdgcn_exp2f(d * 1.44269504088896340736f) - 1.0f;
}

// what is given of a pixel (read before its costs are worked on)
struct MrfPixel {
    int label;
    bool counts;
    float advantage, old_logp, ref_logp;
};

template <bool TRAIN> __device__ inline MrfPixel mrf_policy_pixel(const MrfPolicyParams &P, long long i, bool there)
{
    MrfPixel x = {0, there, 0.0f, 0.0f, 0.0f};
    if (!there) return x;
    x.label = mrf_policy_label(P, i);
    if constexpr (TRAIN) {
        x.counts = !P.mask || P.mask[i] != 0;
        x.advantage = P.advantage[P.per == 1u ? (unsigned)i : (unsigned)i / P.per];
        if (P.old_logp) x.old_logp = P.old_logp[i];
        if (P.ref_logp) x.ref_logp = P.ref_logp[i];
    }
    return x;
}

// what a pixel adds to the two sums, and the slope of the loss in its log-probability (before 1 / n)
__device__ inline void mrf_policy_terms(const MrfPolicyParams &P, const MrfPixel &x, float lp, float &gain, float &div, float &slope)
{
    // (a label that is not allowed: r = 0 and an infinite d, also where the earlier or the reference costs did not allow it either)
    const bool barred = lp == -INFINITY;
    const float over = barred && x.old_logp == lp ? lp : lp - x.old_logp;
    const float r = P.old_logp ? __builtin_amdgcn_exp2f(over * 1.44269504088896340736f) : 1.0f;
    const float open = r * x.advantage, held = fminf(fmaxf(r, P.low), P.high) * x.advantage;
    const bool clipped = open > held;      // (not where either is NaN, which so reaches the loss)
    gain = clipped ? held : open;
    slope = clipped ? 0.0f : -open;
    div = 0.0f;
    if (P.ref_logp) {
        const float d = barred && x.ref_logp == lp ? INFINITY : x.ref_logp - lp, em = mrf_exp_minus_1(d);
        div = em < INFINITY ? em - d : em;      // (a label that is not allowed: infinite, not infinity less infinity)
        if (P.kl > 0.0f) slope -= P.kl * em;
    }
}

// counted pixels among n entries of the mask, for this thread's share of `threads` (16 entries a load where the address allows it)
__device__ inline int mrf_policy_count_share(const uint8_t *mask, long long n, long long thread, long long threads)
{
    int c = 0;
    long long done = 0;
    if (((uintptr_t)mask & 15) == 0) {
        done = n & ~15LL;
        for (long long k = thread * 16; k < done; k += threads * 16) {
            typedef unsigned quad __attribute__((ext_vector_type(4)));
            const quad v = *(const quad *)(mask + k);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // the highest bit of every byte that is not 0
                const unsigned w = v[j];
                c += __popc((((w & 0x7f7f7f7fu) + 0x7f7f7f7fu) | w) & 0x80808080u);
            }
        }
    }
    for (long long k = done + thread; k < n; k += threads) c += mask[k] != 0;
    return c;
}

__device__ inline long long mrf_policy_lanes_count(long long c)
{
    for (int m = 1; m < 64; m <<= 1) c += __shfl_xor(c, m);
    return c;
}

__global__ void __launch_bounds__(256) mrf_policy_count(const MrfPolicyParams P)
{
    __shared__ long long waves[4];
    const long long c = mrf_policy_lanes_count(mrf_policy_count_share(P.mask, P.N, (long long)blockIdx.x * 256 + threadIdx.x, (long long)gridDim.x * 256));
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = c;
    __syncthreads();
    if (threadIdx.x == 0) P.counts[blockIdx.x] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
}

// Number of counted pixels, at least 1, from the counts of `blocks` workgroups, or from the mask itself where there are none (a
// launch of one workgroup); every thread of the workgroup calls it.
__device__ inline long long mrf_policy_counted(const MrfPolicyParams &P, int blocks)
{
    __shared__ long long total[16];
    if (!P.mask) return P.N > 0 ? P.N : 1;
    long long c = 0;
    if (blocks == 0) c = mrf_policy_count_share(P.mask, P.N, threadIdx.x, blockDim.x);
    else
        for (int k = threadIdx.x; k < blocks; k += blockDim.x) c += P.counts[k];
    c = mrf_policy_lanes_count(c);
    if ((threadIdx.x & 63) == 0) total[threadIdx.x >> 6] = c;
    __syncthreads();
    c = 0;
    for (int w = 0; w < (int)(blockDim.x >> 6); ++w) c += total[w];
    return c > 0 ? c : 1;
}

__device__ inline void mrf_policy_loss(const MrfPolicyParams &P, double gain, double div, long long n)
{
    gain /= (double)n;
    div /= (double)n;
    P.loss[0] = (float)(P.kl > 0.0f ? (double)P.kl * div - gain : -gain);
    P.loss[1] = (float)-gain;
    P.loss[2] = (float)div;
}

// factor on the slopes of the pixels
__device__ inline float mrf_policy_factor(const MrfPolicyParams &P, long long n) { return P.scale * (P.upstream ? *P.upstream : 1.0f) / (float)n; }

// what a wavefront's rows add to the two sums ends as one partial sum per workgroup, or as the loss where there is only one (nothing where
// the gradient alone is asked for)
__device__ inline void mrf_policy_partial(const MrfPolicyParams &P, double gain, double div, long long n)
{
    __shared__ double sums[2][16];
    if (!P.loss) return;
    gain = mrf_wave_sum_f64(gain);
    div = mrf_wave_sum_f64(div);
    if ((threadIdx.x & 63) == 0) {
        sums[0][threadIdx.x >> 6] = gain;
        sums[1][threadIdx.x >> 6] = div;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        gain = div = 0.0;
        for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
            gain += sums[0][w];
            div += sums[1][w];
        }
        if (gridDim.x == 1) {
            mrf_policy_loss(P, gain, div, n);
        } else {
            P.partial[2 * (size_t)blockIdx.x] = gain;
            P.partial[2 * (size_t)blockIdx.x + 1] = div;
        }
    }
}

// A row of costs c (infinite behind its end) becomes the exponentials of their distance from the smallest; returns their sum, and the
// smallest.  A row without an allowed label gives zeros.
template <class Row, int E, class Min, class Sum> __device__ inline float mrf_policy_exponentials(float (&c)[E], float &low, Min min, Sum sum)
{
    float v = INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) v = fminf(v, c[e]);
    low = min(v);
    const float from = low < INFINITY ? low : 0.0f;
    v = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        c[e] = mrf_exp_small(from - c[e]);
        v += c[e];
    }
    return sum(v);
}

// Log-probability of the label whose cost is `ca`, from the row's smallest cost and sum (at least 1: the hardware's logarithm to base 2 is off by
// an ulp of it); -infinity where no label is allowed
__device__ inline float mrf_policy_logp(float low, float ca, float s)
{
    return s == 0.0f ? -INFINITY : (low - ca) - __builtin_amdgcn_logf(s) * 0.69314718055994530942f;
}

// ---- rows in registers (MrfRow): one reading of the costs, one writing of the gradient.  About 12 operations a cost, one of them an exponential: bound by
// memory.  2,047 rows of 32,000 in 16 bits 65 us (4.1 TB/s: eight rows a compute unit, and the last ones leave some idle), log-probabilities
// of 116,313 rows of 70 in 32 bits 9 us (3.6 TB/s).
constexpr int mrf_policy_threads(int TL) { return TL <= 256 ? 256 : TL; }

// rows of a lane that are on their way at once (200,000 pixels of 400 labels in 16 bits 92 us, 100 with one; 32 bits the same either way)
constexpr int mrf_policy_batch(int E) { return E <= 4 ? 4 : (E <= 12 ? 2 : 1); }

template <class T, bool TRAIN, int TL, int V, int CH>
__global__ void __launch_bounds__(mrf_policy_threads(TL)) mrf_policy_rows(const MrfPolicyParams P, int count_blocks)
{
    typedef MrfRow<TL, V, CH> Row;
    constexpr int NT = mrf_policy_threads(TL), G = NT / TL, U = TL <= 64 ? mrf_policy_batch(Row::E) : 1;
    __shared__ float scratch[2][NT / 64];
    const int l = threadIdx.x % TL, L = P.L;
    const unsigned group = threadIdx.x / TL, mine = group * (unsigned)L;
    const long long counted = TRAIN ? mrf_policy_counted(P, count_blocks) : 1;
    const float inv_n = TRAIN ? mrf_policy_factor(P, counted) : 0.0f;
    double total_gain = 0.0, total_div = 0.0;
    const long long step = (long long)gridDim.x * G;

    // a row whose costs are `c`
    const auto finish = [&](float (&c)[Row::E], const MrfPixel &pixel, float own, const long long first, bool there) {
        const long long i = first + group;
        float low;
        if (TRAIN && P.mask) {
            // (costs of pixels that do not count may be anything)
#pragma unroll
            for (int e = 0; e < Row::E; ++e) c[e] = pixel.counts ? c[e] : 0.0f;
        }
        const float s = mrf_policy_exponentials<Row>(c, low, [&](float v) { return Row::min(v, scratch[0]); },
                                                     [&](float v) { return Row::sum(v, scratch[1]); });
        const float lp = mrf_policy_logp(low, own, s);
        if (P.logp && there && l == 0) P.logp[i] = pixel.counts ? lp : 0.0f;
        if constexpr (TRAIN) {
            float gain = 0.0f, div = 0.0f, slope = 0.0f;
            const bool adds = pixel.counts && s != 0.0f;
            if (adds) mrf_policy_terms(P, pixel, lp, gain, div, slope);
            if (l == 0) {
                total_gain += (double)gain;
                total_div += (double)div;
            }
            if (P.dcost && there) {
                const float g = slope * inv_n, f = adds ? g / s : 0.0f;
#pragma unroll
                for (int e = 0; e < Row::E; ++e) c[e] *= f;
                T *to = (T *)P.dcost + (size_t)first * L + mine;
                Row::store(to, L, l, c);
                // (the label's entry once more, by the lane that has stored it)
                if (pixel.label / V % TL == l) to[pixel.label] = mrf_from_f32<T>(adds ? f * mrf_exp_small(low - own) - g : 0.0f);
            }
        }
    };
    if constexpr (TL > 64) {
        // long rows: the next one is on its way while this one is worked on
        typename Row::template Raw<T> in;
        MrfPixel pixel;
        const auto fetch = [&](const long long base) {
            const T *at = (const T *)P.cost + (size_t)base * L;
            pixel = mrf_policy_pixel<TRAIN>(P, base + group, base + group < P.N);
            if (mrf_rows_fast(base, G, V, P.N)) Row::template load<true>(at, mine, true, L, l, in);
            else Row::template load<false>(at, mine, base + group < P.N, L, l, in);
        };
        if ((long long)blockIdx.x * G < P.N) fetch((long long)blockIdx.x * G);
        for (long long base = (long long)blockIdx.x * G; base < P.N; base += step) {
            const bool there = base + group < P.N;
            const MrfPixel here = pixel;
            const float own = there ? mrf_to_f32(((const T *)P.cost + (size_t)base * L)[mine + (unsigned)here.label]) : 0.0f;
            float c[Row::E];
            Row::convert(in, L, l, c, INFINITY);
            if (base + step < P.N) fetch(base + step);
            finish(c, here, own, base, there);
        }
    } else {
        const auto rows = [&](auto fast, auto batch, const long long base) {
            constexpr bool FAST = decltype(fast)::value;
            constexpr int n = decltype(batch)::value;
            typename Row::template Raw<T> in[n];
            MrfPixel pixel[n];
            float own[n];
#pragma unroll
            for (int u = 0; u < n; ++u) {
                const long long i = base + u * step + group;
                pixel[u] = mrf_policy_pixel<TRAIN>(P, i, FAST || i < P.N);
            }
#pragma unroll
            for (int u = 0; u < n; ++u) {
                const long long first = base + u * step;
                const bool there = FAST || first + group < P.N;
                const T *at = (const T *)P.cost + (size_t)first * L;
                Row::template load<FAST>(at, mine, there, L, l, in[u]);
                own[u] = there ? mrf_to_f32(at[mine + (unsigned)pixel[u].label]) : 0.0f;
            }
#pragma unroll
            for (int u = 0; u < n; ++u) {
                const long long first = base + u * step;
                float c[Row::E];
                Row::convert(in[u], L, l, c, INFINITY);
                finish(c, pixel[u], own[u], first, FAST || first + group < P.N);
            }
        };
        for (long long base = (long long)blockIdx.x * G; base < P.N;) {
            if (U > 1 && mrf_rows_fast(base + (U - 1) * step, G, V, P.N)) {
                rows(std::true_type{}, std::integral_constant<int, U>{}, base);
                base += U * step;
            } else {
                if (mrf_rows_fast(base, G, V, P.N)) rows(std::true_type{}, std::integral_constant<int, 1>{}, base);
                else rows(std::false_type{}, std::integral_constant<int, 1>{}, base);
                base += step;
            }
        }
    }
    if constexpr (TRAIN) mrf_policy_partial(P, total_gain, total_div, counted);
}

// The same for short rows through LDS (MrfTile): 1,048,576 x 21 in 32 bits, one advantage per image, masked, 39 us (4.9 TB/s).
template <class T, bool TRAIN, int TL, int E>
__global__ void __launch_bounds__(256) mrf_policy_tile(const MrfPolicyParams P, int count_blocks)
{
    typedef MrfTile<TL, E> Tile;
    __shared__ __align__(16) char lds[4][Tile::BYTES];
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, l = lane % TL, g = lane / TL, L = P.L;
    const long long counted = TRAIN ? mrf_policy_counted(P, count_blocks) : 1;
    const float inv_n = TRAIN ? mrf_policy_factor(P, counted) : 0.0f;
    double total_gain = 0.0, total_div = 0.0;
    T *mine = (T *)lds[wv];
    const long long step = (long long)gridDim.x * 4 * Tile::ROWS;
    for (long long base = ((long long)blockIdx.x * 4 + wv) * Tile::ROWS; base < P.N; base += step) {
        const int rows = P.N - base < Tile::ROWS ? (int)(P.N - base) : Tile::ROWS;
        const long long i = base + g;
        const bool there = g < rows;
        const MrfPixel pixel = mrf_policy_pixel<TRAIN>(P, i, there);
        Tile::fetch((const T *)P.cost + (size_t)base * L, rows, L, mine);
        mrf_wave_lds_fence();
        float c[E], low;
        Tile::take(mine, g, L, l, c, INFINITY);
        const float own = mrf_to_f32(mine[g * L + pixel.label]);
        if (TRAIN && P.mask) {
#pragma unroll
            for (int e = 0; e < E; ++e) c[e] = pixel.counts ? c[e] : 0.0f;
        }
        const float s = mrf_policy_exponentials<Tile>(c, low, [](float v) { return Tile::min(v); }, [](float v) { return Tile::sum(v); });
        const float lp = mrf_policy_logp(low, own, s);
        if (P.logp && there && l == 0) P.logp[i] = pixel.counts ? lp : 0.0f;
        if constexpr (TRAIN) {
            float gain = 0.0f, div = 0.0f, slope = 0.0f;
            const bool adds = pixel.counts && s != 0.0f;
            if (adds) mrf_policy_terms(P, pixel, lp, gain, div, slope);
            if (l == 0) {
                total_gain += (double)gain;
                total_div += (double)div;
            }
            if (P.dcost) {
                const float gs = slope * inv_n, f = adds ? gs / s : 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) c[e] *= f;
                mrf_wave_lds_fence();
                Tile::put(mine, g, L, l, c);
                // (the label's entry once more, by the lane that has put it)
                if (there && pixel.label % TL == l) mine[g * L + pixel.label] = mrf_from_f32<T>(adds ? f * mrf_exp_small(low - own) - gs : 0.0f);
                mrf_wave_lds_fence();
                Tile::flush((T *)P.dcost + (size_t)base * L, rows, L, mine);
            }
        }
        mrf_wave_lds_fence();
    }
    if constexpr (TRAIN) mrf_policy_partial(P, total_gain, total_div, counted);
}

// ---- a workgroup per row of any length.  The first pass keeps a running minimum and the sum under it; the second reads the row again, from the
// caches for the most part.  For rows that no workgroup has registers for: 1,000 rows of 45,000 in 16 bits 54 us (rows of 32,000 102 us where registers take
// 67, 2,047 of them).
template <class T, bool TRAIN>
__global__ void __launch_bounds__(1024) mrf_policy_any(const MrfPolicyParams P, int count_blocks)
{
    constexpr int V = 16 / (int)sizeof(T);
    typedef MrfRow<1024, V, 1> Row;
    typedef typename MrfVec<T, V>::type vec;
    __shared__ float scratch[2][16];
    const int t = threadIdx.x, L = P.L, whole = L / V * V;      // (chunks of V labels, and the labels behind them)
    const long long counted = TRAIN ? mrf_policy_counted(P, count_blocks) : 1;
    const float inv_n = TRAIN ? mrf_policy_factor(P, counted) : 0.0f;
    double total_gain = 0.0, total_div = 0.0;
    for (long long i = blockIdx.x; i < P.N; i += gridDim.x) {
        const T *c = (const T *)P.cost + (size_t)i * L;
        T *dc = TRAIN && P.dcost ? (T *)P.dcost + (size_t)i * L : nullptr;
        const MrfPixel pixel = mrf_policy_pixel<TRAIN>(P, i, true);
        if (!pixel.counts) {
            if (dc)
                for (int k = t; k < L; k += 1024) dc[k] = mrf_from_f32<T>(0.0f);
            if (t == 0 && P.logp) P.logp[i] = 0.0f;
            continue;
        }
        const float own = mrf_to_f32(c[pixel.label]);
        float mn = INFINITY, s = 0.0f;
        const auto take = [&](const float (&v)[V]) {
            float to = mn;
#pragma unroll
            for (int j = 0; j < V; ++j) to = fminf(to, v[j]);
            const float from = to < INFINITY ? to : 0.0f;
            s *= mrf_exp_neg(mn < INFINITY ? from - mn : 0.0f);
#pragma unroll
            for (int j = 0; j < V; ++j) s += mrf_exp_neg(from - v[j]);
            mn = to;
        };
#pragma unroll 4
        for (int k = t * V; k < whole; k += 1024 * V) {
            const vec x = *(const vec *)(c + k);
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = mrf_to_f32((T)x[j]);
            take(v);
        }
        if (whole + t < L) {
            float v[V];
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] = j == 0 ? mrf_to_f32(c[whole + t]) : INFINITY;
            take(v);
        }
        const float low = Row::min(mn, scratch[0]), from = low < INFINITY ? low : 0.0f;
        s = Row::sum(s * mrf_exp_neg(mn < INFINITY ? from - mn : 0.0f), scratch[1]);
        const float lp = mrf_policy_logp(low, own, s);
        if (t == 0 && P.logp) P.logp[i] = lp;
        if constexpr (TRAIN) {
            float gain = 0.0f, div = 0.0f, slope = 0.0f;
            if (s != 0.0f) mrf_policy_terms(P, pixel, lp, gain, div, slope);
            if (t == 0) {
                total_gain += (double)gain;
                total_div += (double)div;
            }
            if (dc) {
                const float g = slope * inv_n, f = s != 0.0f ? g / s : 0.0f;
                const auto entry = [&](float v, int k) { return f * mrf_exp_small(from - v) - (k == pixel.label ? g : 0.0f); };
#pragma unroll 4
                for (int k = t * V; k < whole; k += 1024 * V) {
                    vec x = *(const vec *)(c + k);
#pragma unroll
                    for (int j = 0; j < V; ++j) x[j] = mrf_from_f32<T>(entry(mrf_to_f32((T)x[j]), k + j));
                    *(vec *)(dc + k) = x;
                }
                if (whole + t < L) dc[whole + t] = mrf_from_f32<T>(entry(mrf_to_f32(c[whole + t]), whole + t));
            }
        }
        __syncthreads();
    }
    if constexpr (TRAIN) mrf_policy_partial(P, total_gain, total_div, counted);
}

// The loss from the partial sums: one workgroup, the first 512 threads add every 512th of the first sum, the others of the second.
__global__ void __launch_bounds__(1024) mrf_policy_sum(const MrfPolicyParams P, int blocks, int count_blocks)
{
    static_assert(MRF_POLICY_BLOCKS <= 8 * 512, "partial sums of a thread");
    __shared__ double waves[16];
    const int which = threadIdx.x >> 9;
    double x[8], v = 0.0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = (int)(threadIdx.x & 511) + 512 * i;
        x[i] = k < blocks ? P.partial[2 * (size_t)k + which] : 0.0;
    }
    const long long n = mrf_policy_counted(P, count_blocks);
#pragma unroll
    for (int i = 0; i < 8; ++i) v += x[i];
    v = mrf_wave_sum_f64(v);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum[2] = {0.0, 0.0};
        for (int w = 0; w < 16; ++w) sum[w >> 3] += waves[w];
        mrf_policy_loss(P, sum[0], sum[1], n);
    }
}

using namespace mrf_host;

namespace {

int policy_check(int64_t N, int32_t L, int type, int label_bytes)
{
    if (N < 0 || N > 0x7fffffffLL) return MRF_ERR_BAD_SHAPE;
    if (label_bytes != 1 && label_bytes != 4) return MRF_ERR_BAD_ARGUMENT;
    if (L < 1 || L > LONGEST_ROW || (label_bytes == 1 && L > MRF_MAX_LABELS)) return MRF_ERR_BAD_LABELS;
    return known_type(type) ? MRF_OK : MRF_ERR_BAD_ARGUMENT;
}

// counts the mask where more than one workgroup needs the number: `counts` workgroups' counts
int policy_count(const MrfPolicyParams &P, int blocks, int &counts, hipStream_t st)
{
    counts = 0;
    if (!P.mask || blocks <= 1) return MRF_OK;
    const long long need = (P.N + 4095) / 4096;
    counts = (int)(need < MRF_POLICY_COUNTS ? need : MRF_POLICY_COUNTS);
    hipLaunchKernelGGL(mrf_policy_count, dim3((unsigned)counts), dim3(256), 0, st, P);
    return launch_status("mrf_policy_count");
}

template <class T, bool TRAIN, int TL, int V, int CH> int policy_rows(const MrfPolicyParams &P, int &counts, int &blocks, hipStream_t st)
{
    constexpr int NT = mrf_policy_threads(TL), G = NT / TL;
    const long long need = (P.N + G - 1) / G, most = TL > 64 ? MRF_POLICY_LONG_THREADS / NT : MRF_POLICY_BLOCKS;
    blocks = (int)(need < most ? need : most);
    if (TRAIN) {
        const int rc = policy_count(P, blocks, counts, st);
        if (rc != MRF_OK) return rc;
    }
    hipLaunchKernelGGL((mrf_policy_rows<T, TRAIN, TL, V, CH>), dim3((unsigned)blocks), dim3(NT), 0, st, P, counts);
    return launch_status("mrf_policy_rows");
}

template <class T, bool TRAIN, int TL, int E> int policy_tile(const MrfPolicyParams &P, int &counts, int &blocks, hipStream_t st)
{
    constexpr int G = 4 * MrfTile<TL, E>::ROWS;
    const long long need = (P.N + G - 1) / G;
    blocks = (int)(need < 2048 ? need : 2048);
    if (TRAIN) {
        const int rc = policy_count(P, blocks, counts, st);
        if (rc != MRF_OK) return rc;
    }
    hipLaunchKernelGGL((mrf_policy_tile<T, TRAIN, TL, E>), dim3((unsigned)blocks), dim3(256), 0, st, P, counts);
    return launch_status("mrf_policy_tile");
}

// F(TL, V, CH) for each layout, shortest rows first
#define MRF_POLICY_FEW(F) F(1, 4, 1) F(2, 4, 1)
#define MRF_POLICY_FEW_32(F) F(4, 4, 1) F(8, 4, 1)
#define MRF_POLICY_SHORT(F) F(8, 4, 2) F(8, 4, 3) F(16, 4, 2) F(16, 4, 3) F(16, 4, 4)
// (long rows: 512 threads against 256 or 1,024 for 8,000 and 12,000 labels in 16 bits 33 and 50 us instead of 38 and 59, 4,000 pixels; the
// same in 32 bits)
#define MRF_POLICY_LONG(F) \
    F(64, 4, 2) F(64, 4, 3) F(64, 4, 4) F(64, 4, 6) F(64, 4, 8) F(256, 4, 3) F(256, 4, 4) F(512, 4, 3) F(512, 4, 4) F(512, 4, 6) \
    F(1024, 4, 4) F(1024, 4, 6) F(1024, 4, 8)
#define MRF_POLICY_LONG_16(F) \
    F(64, 8, 1) F(64, 8, 2) F(64, 8, 3) F(64, 8, 4) F(256, 8, 2) F(512, 8, 2) F(512, 8, 3) F(1024, 8, 2) F(1024, 8, 3) F(1024, 8, 4)

// Rows through LDS?  Registers / LDS, 40 million costs:
// With the gradient LDS is faster for rows that are no whole chunks (32 bits, 33 labels 96 / 68 us, 149 71 / 66; 16 bits 70 / 44 and 53 / 41) except the shortest
// (6: 108 / 113 and 77 / 87), and for most others of more than 8 labels, as lanes of a power of two idle less and a pixel's terms are worked out
// by fewer of them: 32 bits, 40 labels 84 / 67, 100 72 / 67; 16 bits 61 / 40 and 52 / 41, 192 43 / 41.  Not where a column's entries share LDS
// banks (32 bits: multiples of 32, 64 67 / 90; 16 bits: powers of two, 64 49 / 84), nor for 32-bit rows so long that both only copy (176 66 / 67).
// Log-probabilities alone write nothing that could be in pieces: LDS up to 60 labels (32 bits: 7 42 / 38, 40 32 / 30, 70 30 / 31, 149 27 / 30; 16 bits: 21 / 17 for 40),
// but for multiples of 16 in 32 bits (16: 36 / 45).
template <bool TRAIN> bool policy_tiles(int L, int bytes)
{
    if (L > MRF_TILES_LONGEST) return false;
    if (!TRAIN) return L <= 60 && (L % 4 != 0 || (L > 8 && (bytes == 2 || L % 16 != 0)));
    if (L % 4 != 0) return L > 6;
    return L > 8 && (bytes == 2 ? L < 64 || (L & (L - 1)) != 0 : L <= 150 && L % 32 != 0);
}

template <class T, bool TRAIN> int policy_any_layout(const MrfPolicyParams &P, int &counts, int &blocks, hipStream_t st)
{
    if (policy_tiles<TRAIN>(P.L, (int)sizeof(T))) {
        // (log-probabilities alone: rows of one or two lanes)
#define MRF_LAUNCH(TL, E) \
        if constexpr (TRAIN || TL <= 2) \
            if (P.L <= TL * E) return policy_tile<T, TRAIN, TL, E>(P, counts, blocks, st);
        MRF_TILES(MRF_LAUNCH)
#undef MRF_LAUNCH
    }
    // (with the gradient, no row of 9 to 16 labels in 32 bits is left, and of 16-bit rows up to 256 only the powers of two)
#define MRF_LAUNCH(TL, V, CH) \
    if constexpr (!TRAIN || !(sizeof(T) == 4 ? TL == 4 : TL <= 16 && CH == 3)) \
        if (P.L <= TL * V * CH) return policy_rows<T, TRAIN, TL, V, CH>(P, counts, blocks, st);
    MRF_POLICY_FEW(MRF_LAUNCH)
    if constexpr (sizeof(T) == 4) {
        MRF_POLICY_FEW_32(MRF_LAUNCH)
    }
    MRF_POLICY_SHORT(MRF_LAUNCH)
    if constexpr (sizeof(T) == 2) {
        MRF_POLICY_LONG_16(MRF_LAUNCH)
    } else {
        MRF_POLICY_LONG(MRF_LAUNCH)
    }
#undef MRF_LAUNCH
    blocks = (int)(P.N < MRF_POLICY_BLOCKS ? P.N : MRF_POLICY_BLOCKS);
    if (TRAIN) {
        const int rc = policy_count(P, blocks, counts, st);
        if (rc != MRF_OK) return rc;
    }
    hipLaunchKernelGGL((mrf_policy_any<T, TRAIN>), dim3((unsigned)blocks), dim3(1024), 0, st, P, counts);
    return launch_status("mrf_policy_any");
}

template <class T> int logp_launch(const MrfPolicyParams &P, hipStream_t st)
{
    int counts = 0, blocks = 0;
    return policy_any_layout<T, false>(P, counts, blocks, st);
}

template <class T> int policy_launch(const MrfPolicyParams &P, hipStream_t st)
{
    int counts = 0, blocks = 0;
    const int rc = policy_any_layout<T, true>(P, counts, blocks, st);
    if (rc != MRF_OK || blocks == 1 || !P.loss) return rc;
    hipLaunchKernelGGL(mrf_policy_sum, dim3(1), dim3(1024), 0, st, P, blocks, counts);
    return launch_status("mrf_policy_sum");
}

int policy_of_type(const MrfPolicyParams &P, int cost_type, hipStream_t st)
{
    if (cost_type == MRF_F32) return policy_launch<float>(P, st);
    return cost_type == MRF_F16 ? policy_launch<mrf_f16>(P, st) : policy_launch<mrf_bf16>(P, st);
}

// Checks of the loss and its gradient, and the parameters that follow from the arguments; `required`: what else must not be NULL.
int policy_arguments(MrfPolicyParams &P, int cost_type, int64_t per, float clip_low, float clip_high, void *workspace, size_t workspace_bytes,
                     const void *required)
{
    const int rc = policy_check(P.N, P.L, cost_type, P.label_bytes);
    if (rc != MRF_OK) return rc;
    if (per < 1 || !(clip_low >= 0.0f) || !(clip_low < 1.0f) || !(clip_high >= 0.0f) || !(clip_high < INFINITY) || !(P.kl >= 0.0f) ||
        !(P.kl < INFINITY) || !(fabsf(P.scale) < INFINITY))
        return MRF_ERR_BAD_ARGUMENT;
    if (!required || !workspace || (P.N > 0 && (!P.cost || !P.labels || !P.advantage)) || (P.kl > 0.0f && P.N > 0 && !P.ref_logp))
        return MRF_ERR_NULL_POINTER;
    if (workspace_bytes < mrf_softmin_policy_workspace_bytes()) return MRF_ERR_WORKSPACE_TOO_SMALL;
    P.per = (unsigned)(per < P.N ? per : (P.N > 0 ? P.N : 1));
    P.low = 1.0f - clip_low;
    P.high = 1.0f + clip_high;
    P.counts = (long long *)workspace;
    P.partial = (double *)((char *)workspace + sizeof(long long) * MRF_POLICY_COUNTS);
    return MRF_OK;
}

}  // namespace

extern "C" {

int mrf_softmin_logp(int64_t n_pixels, int32_t L, const void *cost, int cost_type, const void *labels, int label_bytes, float *logp,
                     void *hip_stream)
{
    const int rc = policy_check(n_pixels, L, cost_type, label_bytes);
    if (rc != MRF_OK) return rc;
    if (n_pixels == 0) return MRF_OK;
    if (!cost || !labels || !logp) return MRF_ERR_NULL_POINTER;
    MrfPolicyParams P = {};
    P.N = n_pixels; P.L = L; P.cost = cost; P.labels = labels; P.label_bytes = label_bytes; P.logp = logp;
    hipStream_t st = (hipStream_t)hip_stream;
    if (cost_type == MRF_F32) return logp_launch<float>(P, st);
    return cost_type == MRF_F16 ? logp_launch<mrf_f16>(P, st) : logp_launch<mrf_bf16>(P, st);
}

size_t mrf_softmin_policy_workspace_bytes(void)
{
    return sizeof(long long) * MRF_POLICY_COUNTS + 2 * sizeof(double) * MRF_POLICY_BLOCKS;
}

int mrf_softmin_policy(int64_t n_pixels, int32_t L, const void *cost, int cost_type, const void *labels, int label_bytes,
                       const float *advantage, int64_t pixels_per_advantage, const float *old_logp, const float *ref_logp,
                       const uint8_t *mask, float clip_low, float clip_high, float kl_weight, float grad_scale, float *loss, float *logp,
                       void *grad_cost, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    MrfPolicyParams P = {};
    P.N = n_pixels; P.L = L; P.cost = cost; P.labels = labels; P.label_bytes = label_bytes; P.advantage = advantage; P.old_logp = old_logp;
    P.ref_logp = ref_logp; P.mask = mask; P.kl = kl_weight; P.scale = grad_scale; P.loss = loss; P.logp = logp; P.dcost = grad_cost;
    const int rc = policy_arguments(P, cost_type, pixels_per_advantage, clip_low, clip_high, workspace, workspace_bytes, loss);
    if (rc != MRF_OK) return rc;
    hipStream_t st = (hipStream_t)hip_stream;
    if (n_pixels == 0) {
        P.mask = nullptr;
        hipLaunchKernelGGL(mrf_policy_sum, dim3(1), dim3(1024), 0, st, P, 0, 0);
        return launch_status("mrf_policy_sum");
    }
    return policy_of_type(P, cost_type, st);
}

int mrf_softmin_policy_backward(int64_t n_pixels, int32_t L, const void *cost, int cost_type, const void *labels, int label_bytes,
                                const float *advantage, int64_t pixels_per_advantage, const float *old_logp, const float *ref_logp,
                                const uint8_t *mask, float clip_low, float clip_high, float kl_weight, const float *grad_loss, void *grad_cost,
                                void *workspace, size_t workspace_bytes, void *hip_stream)
{
    MrfPolicyParams P = {};
    P.N = n_pixels; P.L = L; P.cost = cost; P.labels = labels; P.label_bytes = label_bytes; P.advantage = advantage; P.old_logp = old_logp;
    P.ref_logp = ref_logp; P.mask = mask; P.kl = kl_weight; P.scale = 1.0f; P.upstream = grad_loss; P.dcost = grad_cost;
    const int rc = policy_arguments(P, cost_type, pixels_per_advantage, clip_low, clip_high, workspace, workspace_bytes, grad_loss);
    if (rc != MRF_OK || n_pixels == 0) return rc;
    if (!grad_cost) return MRF_ERR_NULL_POINTER;
    return policy_of_type(P, cost_type, (hipStream_t)hip_stream);
}

}  // extern "C"
