// Norm of queries and keys for each head, and their rotation by position, in one pass, forward and backward (see mrf_head_rotation_forward in the
// header for the formulas).
//
// A head of D entries is D / 2 slots of two entries: those that turn together, and behind them neighbours.  TL lanes share a token, MRF_SLOTS
// slots each, and go through some of its heads: the angles are formed once for all of them.  Some 30 operations an entry: bound by memory.
// Angles: position times frequency is formed and reduced to an eighth of a turn in 64 bits (a position of 10^6 leaves 32 bits no digit of the
// angle behind the point), sine and cosine of the rest by their series.
#include "mrfmp_rows.h"

#include <type_traits>

#define MRF_SLOTS 4
#define MRF_ROTATE_PARTS 1024      // workgroups that sum the parameters' gradients, at most

struct MrfRotateParams {
    long long tokens, T;
    int Hq, Hk, D, half, n_axes, interleaved;      // half: pairs that turn
    int heads, pieces;                             // heads that a group of lanes goes through; groups of a token
    const void *in[2], *dout[2];                   // queries, keys
    long long at_batch[2], at_token[2], at_head[2];
    const float *gamma[2], *inv_freq;
    const int *positions;
    long long position_offset;
    float eps;
    void *out[2];                                  // (gradients of the inputs in the backward pass)
    float *dgamma[2], *partial;                    // [parts][2][D]
    int parts;
};

// sine and cosine of `turns` times 2 pi
__device__ inline void mrf_turn(double turns, float &c, float &s)
{
    const double q = rint(4.0 * turns);
    const float x = (float)((turns - 0.25 * q) * 6.28318530717958647692), x2 = x * x;      // |x| <= pi / 4
    const float sn = x * fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), 1.0f);
    const float cs = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
    const int k = (int)(long long)q & 3;
    const float a = k & 1 ? sn : cs, b = k & 1 ? cs : sn;
    c = k == 1 || k == 2 ? -a : a;
    s = k >= 2 ? -b : b;
}

// The slots of a lane: entries e0(j), e1(j) of slot j.  WHOLE: its slots are of one kind and all there, so that its entries are two runs of
// MRF_SLOTS neighbours.
template <class X, bool WHOLE> struct MrfSlots {
    typedef typename MrfVec<X, MRF_SLOTS>::type vec;
    struct Raw { vec v[2]; };
    int first, half, D;
    bool split, any;

    __device__ inline MrfSlots(const MrfRotateParams &P, int l) : first(l * MRF_SLOTS), half(P.half), D(P.D)
    {
        split = !P.interleaved && first < half;
        any = 2 * first < D;
    }
    // where the entries of slot j lie (WHOLE: of the run that it is in)
    __device__ inline int e0(int j) const { return !interleaved_at(j) ? first + j : 2 * (first + j); }
    __device__ inline int e1(int j) const { return !interleaved_at(j) ? first + j + half : 2 * (first + j) + 1; }
    __device__ inline bool interleaved_at(int j) const { return WHOLE ? !split : !(split && first + j < half); }

    __device__ inline void load(const X *at, bool there, Raw &r) const
    {
#pragma unroll
        for (int j = 0; j < MRF_SLOTS; ++j) r.v[0][j] = r.v[1][j] = (X)0.0f;
        if (!there || !any) return;
        if constexpr (WHOLE) {
            r.v[0] = *(const vec *)(at + (split ? first : 2 * first));
            r.v[1] = *(const vec *)(at + (split ? first + half : 2 * first + MRF_SLOTS));
        } else {
#pragma unroll
            for (int j = 0; j < MRF_SLOTS; ++j) {
                if (e0(j) < D) r.v[0][j] = at[e0(j)];
                if (e1(j) < D) r.v[1][j] = at[e1(j)];
            }
        }
    }
    // a[j], b[j]: the two entries of slot j
    __device__ inline void convert(const Raw &r, float (&a)[MRF_SLOTS], float (&b)[MRF_SLOTS]) const
    {
        float u[2 * MRF_SLOTS];
#pragma unroll
        for (int j = 0; j < MRF_SLOTS; ++j) u[j] = mrf_to_f32((X)r.v[0][j]), u[MRF_SLOTS + j] = mrf_to_f32((X)r.v[1][j]);
#pragma unroll
        for (int j = 0; j < MRF_SLOTS; ++j) {
            a[j] = !WHOLE || split ? u[j] : u[2 * j];
            b[j] = !WHOLE || split ? u[MRF_SLOTS + j] : u[2 * j + 1];
        }
    }
    __device__ inline void store(X *at, bool there, const float (&a)[MRF_SLOTS], const float (&b)[MRF_SLOTS]) const
    {
        if (!there || !any) return;
        if constexpr (WHOLE) {
            vec x, y;
#pragma unroll
            for (int j = 0; j < MRF_SLOTS; ++j) {
                const float low = j % 2 ? b[j / 2] : a[j / 2], high = j % 2 ? b[(MRF_SLOTS + j) / 2] : a[(MRF_SLOTS + j) / 2];
                x[j] = mrf_from_f32<X>(split ? a[j] : low);
                y[j] = mrf_from_f32<X>(split ? b[j] : high);
            }
            *(vec *)(at + (split ? first : 2 * first)) = x;
            *(vec *)(at + (split ? first + half : 2 * first + MRF_SLOTS)) = y;
        } else {
#pragma unroll
            for (int j = 0; j < MRF_SLOTS; ++j) {
                if (e0(j) < D) at[e0(j)] = mrf_from_f32<X>(a[j]);
                if (e1(j) < D) at[e1(j)] = mrf_from_f32<X>(b[j]);
            }
        }
    }
    __device__ inline void parameters(const float *at, float (&a)[MRF_SLOTS], float (&b)[MRF_SLOTS], float fill) const
    {
#pragma unroll
        for (int j = 0; j < MRF_SLOTS; ++j) {
            a[j] = at && e0(j) < D ? at[e0(j)] : fill;
            b[j] = at && e1(j) < D ? at[e1(j)] : fill;
        }
    }
};

// cos and sin of a token's angles (1, 0 in slots that do not turn)
template <class S> __device__ inline void mrf_angles(const MrfRotateParams &P, const S &slots, long long token, float (&c)[MRF_SLOTS], float (&s)[MRF_SLOTS])
{
#pragma unroll
    for (int j = 0; j < MRF_SLOTS; ++j) {
        const int slot = slots.first + j;
        c[j] = 1.0f;
        s[j] = 0.0f;
        if (slot < P.half) {
            const long long at = P.positions ? P.positions[token * P.n_axes + slot / (P.half / P.n_axes)] : token % P.T;
            mrf_turn((double)(at + P.position_offset) * ((double)P.inv_freq[slot] * 0.15915494309189533577), c[j], s[j]);
        }
    }
}

constexpr int MRF_ROTATE_AHEAD = 4;      // heads whose loads are on their way together

template <class X, int TL, bool WHOLE> __global__ void __launch_bounds__(256) mrf_rotate_fwd(const MrfRotateParams P)
{
    typedef MrfSlots<X, WHOLE> Slots;
    const int l = threadIdx.x % TL, heads = P.Hq + P.Hk;
    const Slots slots(P, l);
    const float inv = 1.0f / (float)P.D;
    const long long all = P.tokens * P.pieces;
    for (long long g = (long long)blockIdx.x * (256 / TL) + threadIdx.x / TL; g < all; g += (long long)gridDim.x * (256 / TL)) {
        const long long token = g / P.pieces, batch = token / P.T, t = token - batch * P.T;
        const int h0 = (int)(g - token * P.pieces) * P.heads, h1 = h0 + P.heads < heads ? h0 + P.heads : heads;
        const auto from = [&](int h) {
            const int k = h >= P.Hq;
            return (const X *)P.in[k] + batch * P.at_batch[k] + t * P.at_token[k] + (h - (k ? P.Hq : 0)) * P.at_head[k];
        };
        typename Slots::Raw r[MRF_ROTATE_AHEAD];
        float c[MRF_SLOTS], s[MRF_SLOTS];
        for (int h = h0; h < h1; h += MRF_ROTATE_AHEAD) {
#pragma unroll
            for (int i = 0; i < MRF_ROTATE_AHEAD; ++i) slots.load(h + i < h1 ? from(h + i) : nullptr, h + i < h1, r[i]);
            if (h == h0) mrf_angles(P, slots, token, c, s);
#pragma unroll
            for (int i = 0; i < MRF_ROTATE_AHEAD; ++i) {
                if (h + i >= h1) break;
                const int k = h + i >= P.Hq;
                float a[MRF_SLOTS], b[MRF_SLOTS], ga[MRF_SLOTS], gb[MRF_SLOTS], sum = 0.0f;
                slots.convert(r[i], a, b);
                slots.parameters(P.gamma[k], ga, gb, 1.0f);
#pragma unroll
                for (int j = 0; j < MRF_SLOTS; ++j) sum = fmaf(a[j], a[j], fmaf(b[j], b[j], sum));
                const float rs = rsqrtf(fmaf(mrf_lanes_sum<TL>(sum), inv, P.eps));
#pragma unroll
                for (int j = 0; j < MRF_SLOTS; ++j) {
                    const float x = a[j] * rs * ga[j], y = b[j] * rs * gb[j];
                    a[j] = fmaf(x, c[j], -(y * s[j]));
                    b[j] = fmaf(x, s[j], y * c[j]);
                }
                slots.store((X *)P.out[k] + (token * (k ? P.Hk : P.Hq) + h + i - (k ? P.Hq : 0)) * (long long)P.D, true, a, b);
            }
        }
    }
}

// Backward: u = dy turned back, a = u gamma, dx = r (a - h mean(a h)) with h = x r.  The sums of u h stay in registers over all tokens of a group.
template <class X, int TL, bool WHOLE> __global__ void __launch_bounds__(256) mrf_rotate_bwd(const MrfRotateParams P)
{
    typedef MrfSlots<X, WHOLE> Slots;
    __shared__ float lds[4][2][2 * MRF_SLOTS * TL];
    const int l = threadIdx.x % TL, heads = P.Hq + P.Hk;
    const Slots slots(P, l);
    const float inv = 1.0f / (float)P.D;
    float sa[2][MRF_SLOTS] = {}, sb[2][MRF_SLOTS] = {};
    const long long all = P.tokens * P.pieces;
    for (long long g = (long long)blockIdx.x * (256 / TL) + threadIdx.x / TL; g < all; g += (long long)gridDim.x * (256 / TL)) {
        const long long token = g / P.pieces, batch = token / P.T, t = token - batch * P.T;
        const int h0 = (int)(g - token * P.pieces) * P.heads, h1 = h0 + P.heads < heads ? h0 + P.heads : heads;
        const auto dense = [&](int h) { return (token * (h >= P.Hq ? P.Hk : P.Hq) + h - (h >= P.Hq ? P.Hq : 0)) * (long long)P.D; };
        const auto from = [&](int h) {
            const int k = h >= P.Hq;
            return (const X *)P.in[k] + batch * P.at_batch[k] + t * P.at_token[k] + (h - (k ? P.Hq : 0)) * P.at_head[k];
        };
        typename Slots::Raw r[MRF_ROTATE_AHEAD], d[MRF_ROTATE_AHEAD];
        float c[MRF_SLOTS], s[MRF_SLOTS];
        for (int h = h0; h < h1; h += MRF_ROTATE_AHEAD) {
#pragma unroll
            for (int i = 0; i < MRF_ROTATE_AHEAD; ++i) {
                const bool there = h + i < h1;
                slots.load(there ? from(h + i) : nullptr, there, r[i]);
                slots.load(there ? (const X *)P.dout[h + i >= P.Hq] + dense(h + i) : nullptr, there, d[i]);
            }
            if (h == h0) mrf_angles(P, slots, token, c, s);
#pragma unroll
            for (int i = 0; i < MRF_ROTATE_AHEAD; ++i) {
                if (h + i >= h1) break;
                const int k = h + i >= P.Hq;
                float a[MRF_SLOTS], b[MRF_SLOTS], ga[MRF_SLOTS], gb[MRF_SLOTS], da[MRF_SLOTS], db[MRF_SLOTS], sum = 0.0f, along = 0.0f;
                slots.convert(r[i], a, b);
                slots.convert(d[i], da, db);
                slots.parameters(P.gamma[k], ga, gb, 1.0f);
#pragma unroll
                for (int j = 0; j < MRF_SLOTS; ++j) {
                    const float u = fmaf(da[j], c[j], db[j] * s[j]), v = fmaf(db[j], c[j], -(da[j] * s[j]));
                    sum = fmaf(a[j], a[j], fmaf(b[j], b[j], sum));
                    da[j] = u;
                    db[j] = v;
                    along = fmaf(u * ga[j], a[j], fmaf(v * gb[j], b[j], along));
                }
                const float rs = rsqrtf(fmaf(mrf_lanes_sum<TL>(sum), inv, P.eps)), m = mrf_lanes_sum<TL>(along) * inv * rs * rs;
#pragma unroll
                for (int j = 0; j < MRF_SLOTS; ++j) {
                    const float u = da[j], v = db[j];
                    da[j] = rs * fmaf(-m, a[j], u * ga[j]);
                    db[j] = rs * fmaf(-m, b[j], v * gb[j]);
                    const float wa = u * (a[j] * rs), wb = v * (b[j] * rs);
                    sa[0][j] += k ? 0.0f : wa;
                    sb[0][j] += k ? 0.0f : wb;
                    sa[1][j] += k ? wa : 0.0f;
                    sb[1][j] += k ? wb : 0.0f;
                }
                if (P.out[k]) slots.store((X *)P.out[k] + dense(h + i), true, da, db);
            }
        }
    }
    if (!P.partial) return;
    // lanes of a wavefront with the same slots, then its wavefronts
    const int wv = threadIdx.x >> 6;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < MRF_SLOTS; ++j) {
            float x = sa[k][j], y = sb[k][j];
            for (int w = TL; w < 64; w *= 2) {
                x += __shfl_xor(x, w);
                y += __shfl_xor(y, w);
            }
            if ((threadIdx.x & 63) < TL) {
                lds[wv][k][(2 * j) * TL + l] = x;
                lds[wv][k][(2 * j + 1) * TL + l] = y;
            }
        }
    __syncthreads();
    if (threadIdx.x >= TL || !slots.any) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float *const to = P.partial + ((size_t)blockIdx.x * 2 + k) * P.D;
#pragma unroll
        for (int j = 0; j < MRF_SLOTS; ++j)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int n = (2 * j + e) * TL + l, column = e ? slots.e1(j) : slots.e0(j);
                if (column < P.D) to[column] = (lds[0][k][n] + lds[1][k][n]) + (lds[2][k][n] + lds[3][k][n]);
            }
    }
}

__global__ void __launch_bounds__(1024) mrf_rotate_sum(const MrfRotateParams P)
{
    __shared__ float part[64][17];
    const int w = threadIdx.x % 16, s = threadIdx.x / 16, column = blockIdx.x * 16 + w;      // of 2 D
    float v = 0.0f;
    if (column < 2 * P.D)
        for (int p = s; p < P.parts; p += 64) v += P.partial[(size_t)p * 2 * P.D + column];
    part[s][w] = v;
    __syncthreads();
    for (int d = 32; d > 0; d /= 2) {
        if (s < d) part[s][w] += part[s + d][w];
        __syncthreads();
    }
    if (s == 0 && column < 2 * P.D) {
        float *const to = P.dgamma[column >= P.D];
        if (to) to[column >= P.D ? column - P.D : column] = part[0][w];
    }
}

namespace mrf_host {

static int rotate_lanes(int D)
{
    const int slots = (D + 1) / 2, lanes = (slots + MRF_SLOTS - 1) / MRF_SLOTS;
    int TL = 1;
    while (TL < lanes) TL *= 2;
    return TL;
}

template <bool FORWARD, class X, int TL> static int rotate_go(const MrfRotateParams &P, bool whole, unsigned grid, hipStream_t st)
{
    if constexpr (FORWARD) {
        if (whole) mrf_rotate_fwd<X, TL, true><<<grid, 256, 0, st>>>(P);
        else mrf_rotate_fwd<X, TL, false><<<grid, 256, 0, st>>>(P);
        return launch_status("mrf_rotate_fwd");
    } else {
        if (whole) mrf_rotate_bwd<X, TL, true><<<grid, 256, 0, st>>>(P);
        else mrf_rotate_bwd<X, TL, false><<<grid, 256, 0, st>>>(P);
        if (P.partial) mrf_rotate_sum<<<(2 * P.D + 15) / 16, 1024, 0, st>>>(P);
        return launch_status("mrf_rotate_bwd");
    }
}

template <bool FORWARD, class X> static int rotate_typed(MrfRotateParams P, hipStream_t st)
{
    const int TL = rotate_lanes(P.D), heads = P.Hq + P.Hk;
    // heads a group: all of a token's where tokens alone keep the card busy (the angles are formed once), else fewer, down to one
    long long want = (262144 + P.tokens * TL - 1) / (P.tokens * TL);      // groups of a token for 1,024 workgroups
    if (want > heads) want = heads;
    P.heads = (int)((heads + want - 1) / want);
    P.pieces = (heads + P.heads - 1) / P.heads;
    const long long all = P.tokens * P.pieces, groups = (all + 256 / TL - 1) / (256 / TL);
    const long long most = FORWARD ? 0x7fffffffLL : MRF_ROTATE_PARTS;
    const unsigned grid = (unsigned)(groups < most ? groups : most);
    P.parts = (int)grid;
    // runs of MRF_SLOTS neighbours: pairs that turn and the rest of a head in whole ones
    const bool whole = P.D % (2 * MRF_SLOTS) == 0 && (P.interleaved || P.half % MRF_SLOTS == 0);
    switch (TL) {
        case 1: return rotate_go<FORWARD, X, 1>(P, whole, grid, st);
        case 2: return rotate_go<FORWARD, X, 2>(P, whole, grid, st);
        case 4: return rotate_go<FORWARD, X, 4>(P, whole, grid, st);
        case 8: return rotate_go<FORWARD, X, 8>(P, whole, grid, st);
        case 16: return rotate_go<FORWARD, X, 16>(P, whole, grid, st);
        case 32: return rotate_go<FORWARD, X, 32>(P, whole, grid, st);
        default: return rotate_go<FORWARD, X, 64>(P, whole, grid, st);
    }
}

static size_t rotate_workspace(int D) { return (size_t)MRF_ROTATE_PARTS * 2 * D * sizeof(float); }

static int rotate_sizes(long long B, long long T, long long Hq, long long Hk, long long D)
{
    const long long most = 0x7fffffffLL;
    if (B < 0 || T < 0 || Hq < 0 || Hk < 0 || D < 1 || D > 512 || Hq > 65536 || Hk > 65536) return MRF_ERR_BAD_SHAPE;
    if (B > most || T > most || (B && T > most / B)) return MRF_ERR_BAD_SHAPE;
    return MRF_OK;
}

static int rotate_check(const mrf_head_rotation *h, MrfRotateParams &P)
{
    if (!h) return MRF_ERR_NULL_POINTER;
    const int rc = rotate_sizes(h->B, h->T, h->Hq, h->Hk, h->D);
    if (rc != MRF_OK) return rc;
    if (!known_type(h->type) || !(h->eps > 0.0f) || !(h->eps < INFINITY)) return MRF_ERR_BAD_ARGUMENT;
    if (h->rotary < 0 || h->rotary > h->D || h->rotary % 2 || h->n_axes < 1 || (h->rotary / 2) % h->n_axes) return MRF_ERR_BAD_ARGUMENT;
    if (h->n_axes > 1 && !h->positions && h->rotary) return MRF_ERR_NULL_POINTER;
    if (h->position_offset > 1LL << 40 || h->position_offset < -(1LL << 40)) return MRF_ERR_BAD_ARGUMENT;
    for (int i = 0; i < 3; ++i)
        if (h->q_stride[i] < 0 || h->k_stride[i] < 0) return MRF_ERR_BAD_ARGUMENT;
    P.tokens = (long long)h->B * h->T; P.T = h->T; P.Hq = h->Hq; P.Hk = h->Hk; P.D = h->D; P.half = h->rotary / 2; P.n_axes = h->n_axes;
    P.interleaved = h->interleaved != 0;
    P.in[0] = h->q; P.in[1] = h->k; P.gamma[0] = h->gamma_q; P.gamma[1] = h->gamma_k; P.inv_freq = h->inv_freq;
    P.at_batch[0] = h->q_stride[0]; P.at_token[0] = h->q_stride[1]; P.at_head[0] = h->q_stride[2];
    P.at_batch[1] = h->k_stride[0]; P.at_token[1] = h->k_stride[1]; P.at_head[1] = h->k_stride[2];
    P.positions = h->rotary ? h->positions : nullptr; P.position_offset = h->position_offset; P.eps = h->eps;
    if (P.tokens > 0 && ((h->Hq && !h->q) || (h->Hk && !h->k) || (h->rotary && !h->inv_freq))) return MRF_ERR_NULL_POINTER;
    return MRF_OK;
}

template <bool FORWARD> static int rotate_launch(const MrfRotateParams &P, int type, hipStream_t st)
{
    if (type == MRF_F32) return rotate_typed<FORWARD, float>(P, st);
    return type == MRF_F16 ? rotate_typed<FORWARD, mrf_f16>(P, st) : rotate_typed<FORWARD, mrf_bf16>(P, st);
}

}  // namespace mrf_host

using namespace mrf_host;

extern "C" {

int mrf_head_rotation_forward(const mrf_head_rotation *heads, void *out_q, void *out_k, void *hip_stream)
{
    MrfRotateParams P = {};
    const int rc = rotate_check(heads, P);
    if (rc != MRF_OK || P.tokens == 0 || P.Hq + P.Hk == 0) return rc;
    if ((P.Hq && !out_q) || (P.Hk && !out_k)) return MRF_ERR_NULL_POINTER;
    P.out[0] = out_q; P.out[1] = out_k;
    return rotate_launch<true>(P, heads->type, (hipStream_t)hip_stream);
}

size_t mrf_head_rotation_workspace_bytes(int64_t n_tokens, int32_t Hq, int32_t Hk, int32_t D)
{
    return rotate_sizes(n_tokens, 1, Hq, Hk, D) == MRF_OK ? rotate_workspace(D) : 0;
}

int mrf_head_rotation_backward(const mrf_head_rotation *heads, const void *grad_out_q, const void *grad_out_k, void *grad_q, void *grad_k,
                               float *grad_gamma_q, float *grad_gamma_k, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    MrfRotateParams P = {};
    const int rc = rotate_check(heads, P);
    if (rc != MRF_OK) return rc;
    const bool none = P.tokens == 0 || P.Hq + P.Hk == 0;
    if (!none && ((P.Hq && !grad_out_q) || (P.Hk && !grad_out_k))) return MRF_ERR_NULL_POINTER;
    P.dout[0] = grad_out_q; P.dout[1] = grad_out_k; P.out[0] = grad_q; P.out[1] = grad_k;
    P.dgamma[0] = grad_gamma_q; P.dgamma[1] = grad_gamma_k;
    if (grad_gamma_q || grad_gamma_k) {
        if (!workspace) return MRF_ERR_NULL_POINTER;
        if (workspace_bytes < rotate_workspace(P.D)) return MRF_ERR_WORKSPACE_TOO_SMALL;
        P.partial = (float *)workspace;
        if (none) {      // sums over no tokens
            mrf_rotate_sum<<<(2 * P.D + 15) / 16, 1024, 0, (hipStream_t)hip_stream>>>(P);
            return launch_status("mrf_rotate_sum");
        }
    }
    if (none) return MRF_OK;
    return rotate_launch<false>(P, heads->type, (hipStream_t)hip_stream);
}

}  // extern "C"
