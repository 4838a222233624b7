// Layer norm over the rows of a matrix, forward and backward (see mrf_layer_norm_forward in the header for the formulas).
#include "mrfmp_rows.h"

#include <type_traits>

struct MrfNormParams {
    long long N;
    int C;
    const void *x, *dy;
    const float *gamma, *beta;
    float eps;
    void *y, *dx;
    float *mean, *rstd;          // written forward (may be NULL), read backward
    float *partial;              // [P][2][C] sums of dy h and of dy over a workgroup's rows
    float *dgamma, *dbeta;
    int P;
};

// ---- rows in registers: one reading of x (forward), of x and dy (backward).  The variance is the mean square of the differences from the
// mean, both taken from the registers.  Some 12 operations an element forward and 14 backward: bound by memory.  479,232 x 192 in 32 bits
// 130 to 135 us (5.5 TB/s and more, as a copy), 4,096 x 2,048 in 16 bits 10 us (three times a launch that does nothing).  A group of lanes has one row on its way at a
// time; the other wavefronts of the compute unit are what hides its loads (with up to four rows 1 million of 16 in 32 bits 28 instead of 26 us).
constexpr int mrf_norm_threads(int TL) { return TL <= 256 ? 256 : TL; }

// What the mean of 32 bits is off by, the mean `left` of the differences from it, is small but as large as the contrast of a row far from 0
// (constant rows of 1,000.1 would come out as 0.06): it is taken off the differences, and its square off their mean square (never below 0 but for
// its rounding; NaN stays).  It is a second sum over the row.  Not for 16-bit rows of up to 8,192 columns: where their contrast is small against their
// level, all are multiples of one 2^-11th of it, and a sum of 2^13 of them has room in 32 bits; what the product with 1 / C lost is then what
// is left of the sum (4,096 x 2,048 in 16 bits 10.1 us instead of 10.7 with the second sum; 9.9 with neither).
template <class X> constexpr bool mrf_norm_exact(int longest) { return sizeof(X) == 2 && longest <= 8192; }

__device__ inline float mrf_norm_variance(float square, float left)
{
    const float v = fmaf(-left, left, square);
    return v < 0.0f ? 0.0f : v;
}

template <class X, class Y, int TL, int V, int CH>
__global__ void __launch_bounds__(mrf_norm_threads(TL)) mrf_norm_fwd(const MrfNormParams Q)
{
    typedef MrfRow<TL, V, CH> Row;
    constexpr int NT = mrf_norm_threads(TL), G = NT / TL;
    __shared__ float scratch[NT / 64];
    __shared__ __align__(16) float2 pairs[NT / 64];
    const int l = threadIdx.x % TL, C = Q.C;
    const float inv = 1.0f / (float)C;
    float gamma[Row::E], beta[Row::E], in_row[Row::E];      // (in_row: 1 in the row's columns, 0 behind them)
    Row::load_columns(Q.gamma, C, l, gamma, 1.0f);
    Row::load_columns(Q.beta, C, l, beta, 0.0f);
#pragma unroll
    for (int e = 0; e < Row::E; ++e) in_row[e] = Row::column(l, e / V) + e % V < C ? 1.0f : 0.0f;
    const unsigned group = threadIdx.x / TL, mine = group * (unsigned)C;

    const long long step = (long long)gridDim.x * G;      // rows that a launch takes at once

    const auto rows = [&](auto fast, const long long first) {
        constexpr bool FAST = decltype(fast)::value;
        typename Row::template Raw<X> in;
        Row::template load<FAST>((const X *)Q.x + (size_t)first * C, mine, FAST || first + group < Q.N, C, l, in);
        float x[Row::E];
        Row::convert(in, C, l, x, 0.0f);
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < Row::E; ++e) s += x[e];
        const float total = Row::sum(s, scratch), mu = total * inv;
        float left = 0.0f;
        s = 0.0f;
#pragma unroll
        for (int e = 0; e < Row::E; ++e) {
            x[e] = fmaf(-mu, in_row[e], x[e]);
            if constexpr (!mrf_norm_exact<X>(Row::W)) left += x[e];
            s = fmaf(x[e], x[e], s);
        }
        if constexpr (mrf_norm_exact<X>(Row::W)) {
            left = fmaf(-mu, (float)C, total) * inv;
            s = Row::sum(s, (float *)pairs);
        } else {
            Row::sums(left, s, pairs);
            left *= inv;
        }
        const float rs = rsqrtf(mrf_norm_variance(s * inv, left) + Q.eps), off = -left * rs;
#pragma unroll
        for (int e = 0; e < Row::E; ++e) x[e] = fmaf(fmaf(x[e], rs, off), gamma[e], beta[e]);
        if (FAST || first + group < Q.N) {
            Row::store((Y *)Q.y + (size_t)first * C + mine, C, l, x);
            if (l == 0 && Q.mean) Q.mean[first + group] = mu + left;
            if (l == 0 && Q.rstd) Q.rstd[first + group] = rs;
        }
    };
    for (long long base = (long long)blockIdx.x * G; base < Q.N; base += step) {
        if (mrf_rows_fast(base, G, V, Q.N)) rows(std::true_type{}, base);
        else rows(std::false_type{}, base);
    }
}

// The same for short rows through LDS (MrfTile): 1,048,576 x 21 from 16 bits to 32 in 29 us (4.9 TB/s).
template <class X, class Y, int TL, int E>
__global__ void __launch_bounds__(256) mrf_norm_fwd_tile(const MrfNormParams Q)
{
    typedef MrfTile<TL, E> Tile;
    __shared__ __align__(16) char lds[4][Tile::BYTES];
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, l = lane % TL, g = lane / TL, C = Q.C;
    const float inv = 1.0f / (float)C;
    float gamma[E], beta[E];
    Tile::load_columns(Q.gamma, C, l, gamma, 1.0f);
    Tile::load_columns(Q.beta, C, l, beta, 0.0f);
    const long long step = (long long)gridDim.x * 4 * Tile::ROWS;
    for (long long base = ((long long)blockIdx.x * 4 + wv) * Tile::ROWS; base < Q.N; base += step) {
        const int rows = Q.N - base < Tile::ROWS ? (int)(Q.N - base) : Tile::ROWS;
        Tile::fetch((const X *)Q.x + (size_t)base * C, rows, C, (X *)lds[wv]);
        mrf_wave_lds_fence();
        float x[E];
        Tile::take((const X *)lds[wv], g, C, l, x, 0.0f);
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) s += x[e];
        const float total = Tile::sum(s), mu = total * inv;
        float left = 0.0f;
        s = 0.0f;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            x[e] = Tile::column(l, e) < C ? x[e] - mu : 0.0f;
            if constexpr (!mrf_norm_exact<X>(Tile::W)) left += x[e];
            s = fmaf(x[e], x[e], s);
        }
        left = (mrf_norm_exact<X>(Tile::W) ? fmaf(-mu, (float)C, total) : Tile::sum(left)) * inv;
        const float rs = rsqrtf(mrf_norm_variance(Tile::sum(s) * inv, left) + Q.eps), off = -left * rs;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = fmaf(fmaf(x[e], rs, off), gamma[e], beta[e]);
        mrf_wave_lds_fence();
        Tile::put((Y *)lds[wv], g, C, l, x);
        mrf_wave_lds_fence();
        Tile::flush((Y *)Q.y + (size_t)base * C, rows, C, (const Y *)lds[wv]);
        if (l == 0 && g < rows && Q.mean) Q.mean[base + g] = mu + left;
        if (l == 0 && g < rows && Q.rstd) Q.rstd[base + g] = rs;
        mrf_wave_lds_fence();
    }
}

// sum over the lanes of a wavefront that are a multiple of TL apart, in all of them
template <int TL> __device__ inline float mrf_norm_across(float v)
{
    if constexpr (TL <= 1) v += mrf_dpp_f32<0x121>(v);       // row_ror:1
    if constexpr (TL <= 2) v += mrf_dpp_f32<0x122>(v);       // row_ror:2
    if constexpr (TL <= 4) v += mrf_dpp_f32<0x124>(v);       // row_ror:4
    if constexpr (TL <= 8) v += mrf_dpp_f32<0x128>(v);       // row_ror:8
    if constexpr (TL <= 16) v = mrf_xor16_f32(v, true);
    if constexpr (TL <= 32) v = mrf_xor32_f32(v, true);
    return v;
}

constexpr int mrf_norm_bwd_threads(int TL) { return TL <= 64 ? 512 : 1024; }

// The sums over rows stay in registers while a workgroup goes through its rows, and end as one partial sum per workgroup and column: x and dy are read
// once, and no column is summed in an order that depends on the run.  Bound by memory: 1,048,576 x 21 (x in 16 bits, dy in 32) 40 us (4.7 TB/s; rows of
// LDS tiles 55), 4,096 x 2,048 in 16 bits 16 us and 3.9 for the sum over workgroups: a row of a workgroup passes two barriers one after the other, and nothing
// of the next row is on its way meanwhile.
template <class X, class Y, int TL, int V, int CH>
__global__ void __launch_bounds__(mrf_norm_bwd_threads(TL)) mrf_norm_bwd(const MrfNormParams Q)
{
    typedef MrfRow<TL, V, CH> Row;
    constexpr int NT = mrf_norm_bwd_threads(TL), G = NT / TL, SLOTS = TL < 64 ? NT / 64 : G;
    __shared__ float scratch[2][NT / 64];
    __shared__ float share[SLOTS > 1 ? SLOTS * Row::W : 1];
    const int l = threadIdx.x % TL, C = Q.C;
    const float inv = 1.0f / (float)C;
    constexpr bool KEEP = TL < 1024 || Row::E <= 8;      // (else the weight is read again for every row: there are no registers for it)
    float gamma[KEEP ? Row::E : 1], sg[Row::E], sb[Row::E];
    if constexpr (KEEP) Row::load_columns(Q.gamma, C, l, gamma, 1.0f);
#pragma unroll
    for (int e = 0; e < Row::E; ++e) sg[e] = sb[e] = 0.0f;
    const unsigned group = threadIdx.x / TL, mine = group * (unsigned)C;

    const long long step = (long long)gridDim.x * G;

    const auto rows = [&](auto fast, const long long first) {
        constexpr bool FAST = decltype(fast)::value;
        const bool there = FAST || first + group < Q.N;
        typename Row::template Raw<X> in;
        typename Row::template Raw<Y> grad;
        Row::template load<FAST>((const X *)Q.x + (size_t)first * C, mine, there, C, l, in);
        Row::template load<FAST>((const Y *)Q.dy + (size_t)first * C, mine, there, C, l, grad);
        const float mu = there ? Q.mean[first + group] : 0.0f, rs = there ? Q.rstd[first + group] : 0.0f;
        float x[Row::E], dy[Row::E];
        Row::convert(in, C, l, x, 0.0f);
        Row::convert(grad, C, l, dy, 0.0f);
        float sa = 0.0f, sh = 0.0f;
        // (behind a row's end, and behind the last row, dy is 0: nothing is added)
#pragma unroll
        for (int e = 0; e < Row::E; ++e) {
            x[e] = (x[e] - mu) * rs;
            sg[e] = fmaf(dy[e], x[e], sg[e]);
            sb[e] += dy[e];
        }
        if constexpr (KEEP) {
#pragma unroll
            for (int e = 0; e < Row::E; ++e) dy[e] *= gamma[e];
        } else if (Q.gamma) {
            Row::scale_columns(Q.gamma, C, l, dy);
        }
#pragma unroll
        for (int e = 0; e < Row::E; ++e) {
            sa += dy[e];
            sh = fmaf(dy[e], x[e], sh);
        }
        sa = Row::sum(sa, scratch[0]) * inv;
        sh = Row::sum(sh, scratch[1]) * inv;
#pragma unroll
        for (int e = 0; e < Row::E; ++e) dy[e] = rs * (dy[e] - sa - x[e] * sh);
        if (Q.dx && there) Row::store((X *)Q.dx + (size_t)first * C + mine, C, l, dy);
    };
    for (long long base = (long long)blockIdx.x * G; base < Q.N; base += step) {
        if (mrf_rows_fast(base, G, V, Q.N)) rows(std::true_type{}, base);
        else rows(std::false_type{}, base);
    }
    if (!Q.partial) return;
    // the groups' sums of all columns meet in LDS, those of the weight first; a launch of one workgroup then has the whole sums
    const bool whole = gridDim.x == 1;
    float *partial = Q.partial + (size_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *out = whole ? (which ? Q.dbeta : Q.dgamma) : partial + (which ? C : 0);
        if (!out) continue;      // (for the whole workgroup)
        const int slot = TL < 64 ? threadIdx.x >> 6 : threadIdx.x / TL;
#pragma unroll
        for (int e = 0; e < Row::E; ++e) {
            const int c = Row::column(l, e / V) + e % V;
            const float v = mrf_norm_across<TL>(which ? sb[e] : sg[e]);
            if constexpr (SLOTS == 1) {
                if (c < C) out[c] = v;
            } else if (TL >= 64 || (threadIdx.x & 63) < TL) {
                share[slot * Row::W + c] = v;
            }
        }
        if constexpr (SLOTS > 1) {
            __syncthreads();
            for (int c = threadIdx.x; c < C; c += NT) {
                float t = share[c];
#pragma unroll
                for (int w = 1; w < SLOTS; ++w) t += share[w * Row::W + c];
                out[c] = t;
            }
            __syncthreads();
        }
    }
}

// ---- a wavefront per row: any length (rows of more than 16,384 columns forward, 12,288 backward, for which a workgroup has no registers).  Three
// readings, the second and third from the caches for the most part: 1,000 rows of 20,000 in 32 bits 345 us forward and 305 backward (198 + 39 + 19 of kernels),
// where 12,000 in registers take 26 and 53.  A lane adds up as many as 2^25 values one after the other: in 64 bits (backward, 1,000 x 20,000 in 16 bits:
// 345 us with sums in 32 bits, 366 in 64, 286 two columns at a time).
template <class X, class Y>
__global__ void __launch_bounds__(256) mrf_norm_fwd_any(const MrfNormParams Q)
{
    const int lane = threadIdx.x & 63;
    const long long step = (long long)gridDim.x * 4;
    for (long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); r < Q.N; r += step) {
        const X *x = (const X *)Q.x + (size_t)r * Q.C;
        Y *y = (Y *)Q.y + (size_t)r * Q.C;
        double s = 0.0;
        for (int c = lane; c < Q.C; c += 64) s += (double)mrf_to_f32(x[c]);
        const double mean = mrf_wave_sum_f64(s) / (double)Q.C;
        // (differences from the mean in two steps: what its rounding to 32 bits leaves is taken off as well)
        const float mu = (float)mean, left = (float)(mean - (double)mu);
        s = 0.0;
        for (int c = lane; c < Q.C; c += 64) {
            const float d = (mrf_to_f32(x[c]) - mu) - left;
            s = fma((double)d, (double)d, s);
        }
        const float rs = rsqrtf((float)(mrf_wave_sum_f64(s) / (double)Q.C) + Q.eps);
        for (int c = lane; c < Q.C; c += 64) {
            const float h = ((mrf_to_f32(x[c]) - mu) - left) * rs;
            const float g = Q.gamma ? Q.gamma[c] : 1.0f, b = Q.beta ? Q.beta[c] : 0.0f;
            y[c] = mrf_from_f32<Y>(fmaf(h, g, b));
        }
        if (lane == 0 && Q.mean) Q.mean[r] = mu;
        if (lane == 0 && Q.rstd) Q.rstd[r] = rs;
    }
}

template <class X, class Y>
__global__ void __launch_bounds__(256) mrf_norm_bwd_any(const MrfNormParams Q)
{
    const int lane = threadIdx.x & 63;
    const long long step = (long long)gridDim.x * 4;
    for (long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); r < Q.N; r += step) {
        const X *x = (const X *)Q.x + (size_t)r * Q.C;
        const Y *dy = (const Y *)Q.dy + (size_t)r * Q.C;
        X *dx = (X *)Q.dx + (size_t)r * Q.C;
        const float mu = Q.mean[r], rs = Q.rstd[r];
        double sum_a = 0.0, sum_h = 0.0;
#pragma unroll 2
        for (int c = lane; c < Q.C; c += 64) {
            const float h = (mrf_to_f32(x[c]) - mu) * rs;
            const float a = mrf_to_f32(dy[c]) * (Q.gamma ? Q.gamma[c] : 1.0f);
            sum_a += (double)a;
            sum_h = fma((double)a, (double)h, sum_h);
        }
        const float sa = (float)(mrf_wave_sum_f64(sum_a) / (double)Q.C), sh = (float)(mrf_wave_sum_f64(sum_h) / (double)Q.C);
        for (int c = lane; c < Q.C; c += 64) {
            const float h = (mrf_to_f32(x[c]) - mu) * rs;
            const float a = mrf_to_f32(dy[c]) * (Q.gamma ? Q.gamma[c] : 1.0f);
            dx[c] = mrf_from_f32<X>(rs * (a - sa - h * sh));
        }
    }
}

// sums over rows: grid (columns / 64, P), lane = column, a workgroup takes every P-th run of four rows; longer rows than a launch may have columns in turns
template <class X, class Y>
__global__ void __launch_bounds__(256) mrf_norm_param_any(const MrfNormParams Q)
{
    __shared__ float sums[2][4][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    for (long long first = blockIdx.x * 64LL; first < Q.C; first += gridDim.x * 64LL) {
        const long long c = first + lane;
        float sg = 0.0f, sb = 0.0f;
        if (c < Q.C)
            for (long long r = (long long)blockIdx.y * 4 + wv; r < Q.N; r += (long long)Q.P * 4) {
                const float dy = mrf_to_f32(((const Y *)Q.dy)[(size_t)r * Q.C + c]);
                const float h = (mrf_to_f32(((const X *)Q.x)[(size_t)r * Q.C + c]) - Q.mean[r]) * Q.rstd[r];
                sg = fmaf(dy, h, sg);
                sb += dy;
            }
        sums[0][wv][lane] = sg;
        sums[1][wv][lane] = sb;
        __syncthreads();
        if (wv == 0 && c < Q.C) {
            float *p = Q.partial + (size_t)blockIdx.y * 2 * Q.C + c;
            p[0] = (sums[0][0][lane] + sums[0][1][lane]) + (sums[0][2][lane] + sums[0][3][lane]);
            p[Q.C] = (sums[1][0][lane] + sums[1][1][lane]) + (sums[1][2][lane] + sums[1][3][lane]);
        }
        __syncthreads();
    }
}

// Weight and bias gradients from the P partial sums of a column: 16 columns per workgroup, 64 threads share a column's partial sums
// (thread k takes every 64th from the k-th on) and add up by halves.
__global__ void __launch_bounds__(1024) mrf_norm_param_sum(const MrfNormParams Q)
{
    __shared__ float sums[64][17];
    const int col = threadIdx.x & 15, part = threadIdx.x >> 4;
    for (long long first = blockIdx.x * 16LL; first < 2LL * Q.C; first += gridDim.x * 16LL) {
        const long long c = first + col;      // [0, C) weight, [C, 2 C) bias
        float s = 0.0f;
        if (c < 2LL * Q.C)
#pragma unroll 8
            for (int p = part; p < Q.P; p += 64) s += Q.partial[(size_t)p * 2 * Q.C + c];
        sums[part][col] = s;
        __syncthreads();
#pragma unroll
        for (int half = 32; half > 0; half >>= 1) {
            if (part < half) sums[part][col] += sums[part + half][col];
            __syncthreads();
        }
        if (part == 0 && c < 2LL * Q.C) {
            s = sums[0][col];
            if (c < Q.C) {
                if (Q.dgamma) Q.dgamma[c] = s;
            } else if (Q.dbeta) {
                Q.dbeta[c - Q.C] = s;
            }
        }
    }
}

using namespace mrf_host;

namespace {

// Workgroups of a backward call at most, each of which leaves a partial sum: one for so little that a second launch would take longer than its rows
// (2,048 x 16: 9 us with one, 5.7 us with 16 and a sum of theirs, but 9.7 us from call to call); else two on each compute unit up to 128 columns (1 million of
// 40 in 16 bits 59 us, 83 with one), and one beyond, where the partial sums' own traffic costs more (4,000 of 1,000 16 us, 20 with two; 2,000 of
// 8,600 in 16 bits 46 and 60).
int norm_partials(int64_t n_rows, int32_t C)
{
    const int most = (long long)C * n_rows <= 32768 && C <= 1024 ? 1 : (C <= 128 ? 512 : 256);
    return (int)(most < n_rows ? most : n_rows);
}

// Workgroups for so many runs of columns: a launch has fewer than 2^32 threads along an index, and more than 16,384 workgroups keep no
// more compute units busy.
unsigned norm_grid(long long runs) { return (unsigned)(runs < 16384 ? runs : 16384); }

int norm_check(int64_t n_rows, int32_t C, int x_type, int y_type)
{
    if (n_rows < 0 || n_rows > 0x7fffffffLL || C < 1 || C > LONGEST_ROW) return MRF_ERR_BAD_SHAPE;
    if (!known_type(x_type) || !known_type(y_type) || (y_type != x_type && y_type != MRF_F32)) return MRF_ERR_BAD_ARGUMENT;
    return MRF_OK;
}

template <class X, class Y, int TL, int V, int CH> int norm_fwd_rows(const MrfNormParams &Q, hipStream_t st)
{
    constexpr int NT = mrf_norm_threads(TL), G = NT / TL;
    const long long need = (Q.N + G - 1) / G, most = NT == 256 ? 4096 : 1024;
    hipLaunchKernelGGL((mrf_norm_fwd<X, Y, TL, V, CH>), dim3((unsigned)(need < most ? need : most)), dim3(NT), 0, st, Q);
    return launch_status("mrf_norm_fwd");
}

template <class X, class Y, int TL, int V, int CH> int norm_bwd_rows(const MrfNormParams &Q, hipStream_t st, int &blocks)
{
    constexpr int G = mrf_norm_bwd_threads(TL) / TL;
    const long long need = (Q.N + G - 1) / G;
    blocks = (int)(need < Q.P ? need : Q.P);
    hipLaunchKernelGGL((mrf_norm_bwd<X, Y, TL, V, CH>), dim3((unsigned)blocks), dim3(mrf_norm_bwd_threads(TL)), 0, st, Q);
    return launch_status("mrf_norm_bwd");
}

// F(TL, V, CH) for each layout, shortest rows first.  Forward a lane holds three values per column (x, weight, bias), backward four or five (x,
// dy, two sums, the weight): 16 and 12 columns at most where a workgroup of 1,024 threads leaves 128 registers.
#define MRF_NORM_FWD_SHORT(F) \
    F(1, 4, 1) F(2, 4, 1) F(4, 4, 1) F(8, 4, 1) F(8, 4, 2) F(8, 4, 3) F(16, 4, 2) F(16, 4, 3) F(16, 4, 4)
#define MRF_NORM_FWD_LONG(F) \
    F(64, 4, 2) F(64, 4, 3) F(64, 4, 4) F(256, 4, 2) F(256, 4, 3) F(256, 4, 4) F(256, 4, 6) F(256, 4, 8) F(1024, 4, 3) F(1024, 4, 4)
#define MRF_NORM_FWD_LONG_16(F) F(64, 8, 1) F(64, 8, 2) F(256, 8, 1) F(256, 8, 2) F(256, 8, 3) F(256, 8, 4) F(1024, 8, 2)
#define MRF_NORM_BWD_SHORT(F) F(1, 4, 1) F(2, 4, 1) F(4, 4, 1) F(8, 4, 1) F(8, 4, 2) F(16, 4, 2) F(16, 4, 3) F(16, 4, 4)
#define MRF_NORM_BWD_LONG(F) F(64, 4, 2) F(64, 4, 3) F(64, 4, 4) F(256, 4, 2) F(1024, 4, 1) F(1024, 4, 2) F(1024, 4, 3)
#define MRF_NORM_BWD_LONG_16(F) F(64, 8, 1) F(64, 8, 2) F(256, 8, 1) F(1024, 8, 1) F(1024, 4, 3)

// Forward, rows through LDS: those that are no whole chunks (in 32 bits, registers / LDS: 1 million of 21 44 / 37 us, 300,000 of 149 71 / 68), and those of 20
// to 60 columns, which leave lanes of a power of two idle (1 million of 36: 66 / 59, from 16 bits to 32 60 / 45, in 16 bits 43 / 32; of 20: 37 / 35, 32 / 26,
// 19 / 18), except multiples of 16, whose entries of a column share LDS banks (32: 52 / 122).  Longer whole chunks in registers (262,144 of
// 100 in 16 bits 20 / 28).
bool norm_tiles(int C) { return C <= MRF_TILES_LONGEST && (C % 4 != 0 || (C > 16 && C < 64 && C % 16 != 0)); }

template <class X, class Y, int TL, int E> int norm_fwd_tiles(const MrfNormParams &Q, hipStream_t st)
{
    constexpr int G = 4 * MrfTile<TL, E>::ROWS;
    const long long need = (Q.N + G - 1) / G;
    hipLaunchKernelGGL((mrf_norm_fwd_tile<X, Y, TL, E>), dim3((unsigned)(need < 2048 ? need : 2048)), dim3(256), 0, st, Q);
    return launch_status("mrf_norm_fwd_tile");
}

template <class X, class Y> int norm_forward(const MrfNormParams &Q, hipStream_t st)
{
    if (norm_tiles(Q.C)) {
#define MRF_LAUNCH(TL, E) \
        if (Q.C <= TL * E) return norm_fwd_tiles<X, Y, TL, E>(Q, st);
        MRF_TILES(MRF_LAUNCH)
#undef MRF_LAUNCH
    }
#define MRF_LAUNCH(TL, V, CH) \
    if (Q.C <= TL * V * CH) return norm_fwd_rows<X, Y, TL, V, CH>(Q, st);
    MRF_NORM_FWD_SHORT(MRF_LAUNCH)
    if constexpr (sizeof(X) == 2) {
        MRF_NORM_FWD_LONG_16(MRF_LAUNCH)
    } else {
        MRF_NORM_FWD_LONG(MRF_LAUNCH)
    }
#undef MRF_LAUNCH
    const long long rows = (Q.N + 3) / 4;
    hipLaunchKernelGGL((mrf_norm_fwd_any<X, Y>), dim3((unsigned)(rows < 8192 ? rows : 8192)), dim3(256), 0, st, Q);
    return launch_status("mrf_norm_fwd_any");
}

// `summed`: one workgroup has written the weight's and the bias's gradient itself
template <class X, class Y> int norm_bwd_launch(MrfNormParams &Q, bool &summed, hipStream_t st)
{
#define MRF_LAUNCH(TL, V, CH) \
    if (Q.C <= TL * V * CH) { \
        const int rc = norm_bwd_rows<X, Y, TL, V, CH>(Q, st, Q.P); \
        summed = Q.P == 1; \
        return rc; \
    }
    MRF_NORM_BWD_SHORT(MRF_LAUNCH)
    if constexpr (sizeof(X) == 2) {
        MRF_NORM_BWD_LONG_16(MRF_LAUNCH)
    } else {
        MRF_NORM_BWD_LONG(MRF_LAUNCH)
    }
#undef MRF_LAUNCH
    if (Q.dx) {
        const long long rows = (Q.N + 3) / 4;
        hipLaunchKernelGGL((mrf_norm_bwd_any<X, Y>), dim3((unsigned)(rows < 8192 ? rows : 8192)), dim3(256), 0, st, Q);
        const int rc = launch_status("mrf_norm_bwd_any");
        if (rc != MRF_OK) return rc;
    }
    if (!Q.partial) return MRF_OK;
    hipLaunchKernelGGL((mrf_norm_param_any<X, Y>), dim3(norm_grid((Q.C + 63LL) / 64), (unsigned)Q.P), dim3(256), 0, st, Q);
    return launch_status("mrf_norm_param_any");
}

template <class X, class Y> int norm_backward(MrfNormParams Q, hipStream_t st)
{
    const bool params = Q.dgamma || Q.dbeta;
    if (!params) Q.partial = nullptr;
    if (Q.N > 0 && (params || Q.dx)) {
        bool summed = false;
        const int rc = norm_bwd_launch<X, Y>(Q, summed, st);
        if (rc != MRF_OK || summed) return rc;
    }
    if (!params) return MRF_OK;
    hipLaunchKernelGGL(mrf_norm_param_sum, dim3(norm_grid((2LL * Q.C + 15) / 16)), dim3(1024), 0, st, Q);
    return launch_status("mrf_norm_param_sum");
}

}  // namespace

extern "C" {

size_t mrf_layer_norm_workspace_bytes(int64_t n_rows, int32_t C)
{
    if (norm_check(n_rows, C, MRF_F32, MRF_F32) != MRF_OK) return 0;
    const size_t bytes = sizeof(float) * 2 * (size_t)norm_partials(n_rows, C) * (size_t)C;
    return bytes ? bytes : 256;
}

int mrf_layer_norm_forward(int64_t n_rows, int32_t C, const void *x, int x_type, const float *gamma, const float *beta, float eps,
                           void *y, int y_type, float *mean, float *rstd, void *hip_stream)
{
    const int rc = norm_check(n_rows, C, x_type, y_type);
    if (rc != MRF_OK) return rc;
    if (!(eps > 0.0f) || !(eps < INFINITY)) return MRF_ERR_BAD_ARGUMENT;
    if (n_rows == 0) return MRF_OK;
    if (!x || !y) return MRF_ERR_NULL_POINTER;
    MrfNormParams Q = {};
    Q.N = n_rows; Q.C = C; Q.x = x; Q.gamma = gamma; Q.beta = beta; Q.eps = eps; Q.y = y; Q.mean = mean; Q.rstd = rstd;
    hipStream_t st = (hipStream_t)hip_stream;
    if (x_type == MRF_F32) return norm_forward<float, float>(Q, st);
    if (x_type == MRF_F16) return y_type == MRF_F32 ? norm_forward<mrf_f16, float>(Q, st) : norm_forward<mrf_f16, mrf_f16>(Q, st);
    return y_type == MRF_F32 ? norm_forward<mrf_bf16, float>(Q, st) : norm_forward<mrf_bf16, mrf_bf16>(Q, st);
}

int mrf_layer_norm_backward(int64_t n_rows, int32_t C, const void *grad_y, int y_type, const void *x, int x_type, const float *gamma,
                            const float *mean, const float *rstd, void *grad_x, float *grad_gamma, float *grad_beta, void *workspace,
                            size_t workspace_bytes, void *hip_stream)
{
    const int rc = norm_check(n_rows, C, x_type, y_type);
    if (rc != MRF_OK) return rc;
    if (n_rows > 0 && (!grad_y || !x || !mean || !rstd)) return MRF_ERR_NULL_POINTER;
    if (grad_gamma || grad_beta) {
        if (!workspace) return MRF_ERR_NULL_POINTER;
        if (workspace_bytes < mrf_layer_norm_workspace_bytes(n_rows, C)) return MRF_ERR_WORKSPACE_TOO_SMALL;
    }
    MrfNormParams Q = {};
    Q.N = n_rows; Q.C = C; Q.x = x; Q.dy = grad_y; Q.gamma = gamma; Q.mean = (float *)mean; Q.rstd = (float *)rstd;
    Q.dx = grad_x; Q.dgamma = grad_gamma; Q.dbeta = grad_beta; Q.partial = (float *)workspace; Q.P = norm_partials(n_rows, C);
    hipStream_t st = (hipStream_t)hip_stream;
    if (x_type == MRF_F32) return norm_backward<float, float>(Q, st);
    if (x_type == MRF_F16) return y_type == MRF_F32 ? norm_backward<mrf_f16, float>(Q, st) : norm_backward<mrf_f16, mrf_f16>(Q, st);
    return y_type == MRF_F32 ? norm_backward<mrf_bf16, float>(Q, st) : norm_backward<mrf_bf16, mrf_bf16>(Q, st);
}

}  // extern "C"
