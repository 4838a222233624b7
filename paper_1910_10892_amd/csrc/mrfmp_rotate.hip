// Norm of queries and keys for each head, and their rotation by position, in one pass, forward and backward (see mrf_head_rotation_forward in the
// header for the formulas).
//
// A head of D entries is D / 2 slots of two entries: those that turn together, and behind them neighbours.  TL lanes share a token, S
// slots each, and go through some of its heads of queries, or of keys: the angles are formed once for all of them.  Some 30 operations an entry: bound by memory.
// Angles: position times frequency is formed and reduced to an eighth of a turn in 64 bits (a position of 10^6 leaves 32 bits no digit of the
// angle behind the point), sine and cosine of the rest by their series.  16 + 4 heads of 128 of 8,192 tokens out of one projection, 16 bits: forward 22 us (3.8 TB/s),
// backward 28 (4.5) and 4.7 for the sums of the parameters' gradients (a copy reaches 5.1).
#include "mrfmp_rows.h"

#include <type_traits>

#define MRF_ROTATE_PARTS 512      // workgroups that sum a parameter's gradient, at most

struct MrfRotateParams {
    long long tokens, T;
    int Hq, Hk, D, half, n_axes, interleaved;      // half: pairs that turn
    int heads, pieces[2];                          // heads that a group of lanes goes through; groups of a token, for its queries and its keys
    int blocks[2];                                 // workgroups, of queries first
    const void *in[2], *dout[2];                   // queries, keys
    long long at_batch[2], at_token[2], at_head[2];
    const float *gamma[2], *inv_freq;
    const int *positions;
    long long position_offset;
    float eps;
    void *out[2];                                  // (gradients of the inputs in the backward pass)
    float *dgamma[2], *partial;                    // [2][MRF_ROTATE_PARTS][D]
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
// S neighbours.
template <class X, int S, bool WHOLE> struct MrfSlots {
    typedef typename MrfVec<X, S>::type vec;
    struct Raw { vec v[2]; };
    int first, half, D;
    bool split, any;

    __device__ inline MrfSlots(const MrfRotateParams &P, int l) : first(l * S), half(P.half), D(P.D)
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
        for (int j = 0; j < S; ++j) r.v[0][j] = r.v[1][j] = (X)0.0f;
        if (!there || !any) return;
        if constexpr (WHOLE) {
            r.v[0] = *(const vec *)(at + (split ? first : 2 * first));
            r.v[1] = *(const vec *)(at + (split ? first + half : 2 * first + S));
        } else {
#pragma unroll
            for (int j = 0; j < S; ++j) {
                if (e0(j) < D) r.v[0][j] = at[e0(j)];
                if (e1(j) < D) r.v[1][j] = at[e1(j)];
            }
        }
    }
    // a[j], b[j]: the two entries of slot j
    __device__ inline void convert(const Raw &r, float (&a)[S], float (&b)[S]) const
    {
        float u[2 * S];
#pragma unroll
        for (int j = 0; j < S; ++j) u[j] = mrf_to_f32((X)r.v[0][j]), u[S + j] = mrf_to_f32((X)r.v[1][j]);
#pragma unroll
        for (int j = 0; j < S; ++j) {
            a[j] = !WHOLE || split ? u[j] : u[2 * j];
            b[j] = !WHOLE || split ? u[S + j] : u[2 * j + 1];
        }
    }
    __device__ inline void store(X *at, bool there, const float (&a)[S], const float (&b)[S]) const
    {
        if (!there || !any) return;
        if constexpr (WHOLE) {
            vec x, y;
#pragma unroll
            for (int j = 0; j < S; ++j) {
                const float low = j % 2 ? b[j / 2] : a[j / 2], high = j % 2 ? b[(S + j) / 2] : a[(S + j) / 2];
                x[j] = mrf_from_f32<X>(split ? a[j] : low);
                y[j] = mrf_from_f32<X>(split ? b[j] : high);
            }
            *(vec *)(at + (split ? first : 2 * first)) = x;
            *(vec *)(at + (split ? first + half : 2 * first + S)) = y;
        } else {
#pragma unroll
            for (int j = 0; j < S; ++j) {
                if (e0(j) < D) at[e0(j)] = mrf_from_f32<X>(a[j]);
                if (e1(j) < D) at[e1(j)] = mrf_from_f32<X>(b[j]);
            }
        }
    }
    __device__ inline void parameters(const float *at, float (&a)[S], float (&b)[S], float fill) const
    {
#pragma unroll
        for (int j = 0; j < S; ++j) {
            a[j] = at && e0(j) < D ? at[e0(j)] : fill;
            b[j] = at && e1(j) < D ? at[e1(j)] : fill;
        }
    }
};

// cos and sin of a token's angles (1, 0 in slots that do not turn)
template <int S, class Slots> __device__ inline void mrf_angles(const MrfRotateParams &P, const Slots &slots, long long token, long long t, float (&c)[S], float (&s)[S])
{
#pragma unroll
    for (int j = 0; j < S; ++j) {
        const int slot = slots.first + j;
        c[j] = 1.0f;
        s[j] = 0.0f;
        if (slot < P.half) {
            const long long at = P.positions ? P.positions[token * P.n_axes + (P.n_axes == 1 ? 0 : slot / (P.half / P.n_axes))] : t;
            mrf_turn((double)(at + P.position_offset) * ((double)P.inv_freq[slot] * 0.15915494309189533577), c[j], s[j]);
        }
    }
}

// heads whose loads are on their way together
constexpr int MRF_ROTATE_AHEAD = 2, MRF_ROTATE_AHEAD_BACK = 1;

// Where a group of lanes is: its kind (0: queries, 1: keys), its first piece, and the way to its next one
template <int TL> struct MrfRotatePlace {
    int kind, heads;
    long long g, all, step;
    __device__ inline MrfRotatePlace(const MrfRotateParams &P)
    {
        kind = blockIdx.x >= (unsigned)P.blocks[0];
        heads = kind ? P.Hk : P.Hq;
        all = P.tokens * P.pieces[kind];
        g = (long long)(blockIdx.x - (kind ? P.blocks[0] : 0)) * (256 / TL) + threadIdx.x / TL;
        step = (long long)P.blocks[kind] * (256 / TL);
    }
};

template <class X, int S, int TL, bool WHOLE> __global__ void __launch_bounds__(256) mrf_rotate_fwd(const MrfRotateParams P)
{
    typedef MrfSlots<X, S, WHOLE> Slots;
    const MrfRotatePlace<TL> place(P);
    const int kind = place.kind;
    const Slots slots(P, threadIdx.x % TL);
    const float inv = 1.0f / (float)P.D;
    float ga[S], gb[S];
    slots.parameters(P.gamma[kind], ga, gb, 1.0f);
    for (long long g = place.g; g < place.all; g += place.step) {
        const long long token = g / P.pieces[kind], batch = token / P.T, t = token - batch * P.T;
        const int h0 = (int)(g - token * P.pieces[kind]) * P.heads, h1 = h0 + P.heads < place.heads ? h0 + P.heads : place.heads;
        const X *const from = (const X *)P.in[kind] + batch * P.at_batch[kind] + t * P.at_token[kind];
        X *const to = (X *)P.out[kind] + token * place.heads * (long long)P.D;
        typename Slots::Raw r[MRF_ROTATE_AHEAD];
        float c[S], s[S];
        for (int h = h0; h < h1; h += MRF_ROTATE_AHEAD) {
#pragma unroll
            for (int i = 0; i < MRF_ROTATE_AHEAD; ++i) slots.load(from + (h + i) * P.at_head[kind], h + i < h1, r[i]);
            if (h == h0) mrf_angles<S>(P, slots, token, t, c, s);
#pragma unroll
            for (int i = 0; i < MRF_ROTATE_AHEAD; ++i) {
                if (h + i >= h1) break;
                float a[S], b[S], sum = 0.0f;
                slots.convert(r[i], a, b);
#pragma unroll
                for (int j = 0; j < S; ++j) sum = fmaf(a[j], a[j], fmaf(b[j], b[j], sum));
                const float rs = rsqrtf(fmaf(mrf_lanes_sum<TL>(sum), inv, P.eps));
#pragma unroll
                for (int j = 0; j < S; ++j) {
                    const float x = a[j] * rs * ga[j], y = b[j] * rs * gb[j];
                    a[j] = fmaf(x, c[j], -(y * s[j]));
                    b[j] = fmaf(x, s[j], y * c[j]);
                }
                slots.store(to + (h + i) * (long long)P.D, true, a, b);
            }
        }
    }
}

// Backward: u = dy turned back, a = u gamma, dx = r (a - h mean(a h)) with h = x r.  The sums of u h of a piece's heads are added in 32
// bits, those of a group's pieces in 64 (terms that are all alike are rounded the same way each time: 128 pieces of 16 heads left the sum off by 2e-5).
template <class X, int S, int TL, bool WHOLE> __global__ void __launch_bounds__(256) mrf_rotate_bwd(const MrfRotateParams P)
{
    typedef MrfSlots<X, S, WHOLE> Slots;
    __shared__ float lds[4][2 * S * TL];
    const MrfRotatePlace<TL> place(P);
    const int kind = place.kind, l = threadIdx.x % TL;
    const Slots slots(P, l);
    const float inv = 1.0f / (float)P.D;
    float ga[S], gb[S];
    // A thread's sums, its own.  (In registers they would cost 16 + 4 heads of 128 a wavefront a SIMD: both passes over 8,192 tokens 54 us, and 50 so; 49 with sums of 32 bits.)
    __shared__ double all[2 * S][256];
#pragma unroll
    for (int j = 0; j < 2 * S; ++j) all[j][threadIdx.x] = 0.0;
    slots.parameters(P.gamma[kind], ga, gb, 1.0f);
    for (long long g = place.g; g < place.all; g += place.step) {
        const long long token = g / P.pieces[kind], batch = token / P.T, t = token - batch * P.T;
        const int h0 = (int)(g - token * P.pieces[kind]) * P.heads, h1 = h0 + P.heads < place.heads ? h0 + P.heads : place.heads;
        const X *const from = (const X *)P.in[kind] + batch * P.at_batch[kind] + t * P.at_token[kind];
        const long long dense = token * place.heads * (long long)P.D;
        typename Slots::Raw r[MRF_ROTATE_AHEAD_BACK], d[MRF_ROTATE_AHEAD_BACK];
        float c[S], s[S], sa[S] = {}, sb[S] = {};
        for (int h = h0; h < h1; h += MRF_ROTATE_AHEAD_BACK) {
#pragma unroll
            for (int i = 0; i < MRF_ROTATE_AHEAD_BACK; ++i) {
                slots.load(from + (h + i) * P.at_head[kind], h + i < h1, r[i]);
                slots.load((const X *)P.dout[kind] + dense + (h + i) * (long long)P.D, h + i < h1, d[i]);
            }
            if (h == h0) mrf_angles<S>(P, slots, token, t, c, s);
#pragma unroll
            for (int i = 0; i < MRF_ROTATE_AHEAD_BACK; ++i) {
                if (h + i >= h1) break;
                float a[S], b[S], da[S], db[S], sum = 0.0f, along = 0.0f;
                slots.convert(r[i], a, b);
                slots.convert(d[i], da, db);
#pragma unroll
                for (int j = 0; j < S; ++j) {
                    const float u = fmaf(da[j], c[j], db[j] * s[j]), v = fmaf(db[j], c[j], -(da[j] * s[j]));
                    sum = fmaf(a[j], a[j], fmaf(b[j], b[j], sum));
                    da[j] = u;
                    db[j] = v;
                    along = fmaf(u * ga[j], a[j], fmaf(v * gb[j], b[j], along));
                }
                const float rs = rsqrtf(fmaf(mrf_lanes_sum<TL>(sum), inv, P.eps)), m = mrf_lanes_sum<TL>(along) * inv * rs * rs;
#pragma unroll
                for (int j = 0; j < S; ++j) {
                    const float u = da[j], v = db[j];
                    da[j] = rs * fmaf(-m, a[j], u * ga[j]);
                    db[j] = rs * fmaf(-m, b[j], v * gb[j]);
                    sa[j] = fmaf(u, a[j] * rs, sa[j]);
                    sb[j] = fmaf(v, b[j] * rs, sb[j]);
                }
                if (P.out[kind]) slots.store((X *)P.out[kind] + dense + (h + i) * (long long)P.D, true, da, db);
            }
        }
#pragma unroll
        for (int j = 0; j < S; ++j) {
            unsafeAtomicAdd(&all[2 * j][threadIdx.x], (double)sa[j]);
            unsafeAtomicAdd(&all[2 * j + 1][threadIdx.x], (double)sb[j]);
        }
    }
    if (!P.dgamma[kind]) return;
    // lanes of a wavefront with the same slots, then its wavefronts
    const int wv = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < S; ++j) {
        float x = (float)all[2 * j][threadIdx.x], y = (float)all[2 * j + 1][threadIdx.x];
        for (int w = TL; w < 64; w *= 2) {
            x += __shfl_xor(x, w);
            y += __shfl_xor(y, w);
        }
        if ((threadIdx.x & 63) < TL) {
            lds[wv][(2 * j) * TL + l] = x;
            lds[wv][(2 * j + 1) * TL + l] = y;
        }
    }
    __syncthreads();
    if (threadIdx.x >= TL || !slots.any) return;
    const bool one = P.blocks[kind] == 1;      // (a single workgroup's sums are all there is)
    float *const to = one ? P.dgamma[kind] : P.partial + ((size_t)kind * MRF_ROTATE_PARTS + blockIdx.x - (kind ? P.blocks[0] : 0)) * P.D;
#pragma unroll
    for (int j = 0; j < S; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int n = (2 * j + e) * TL + l, column = e ? slots.e1(j) : slots.e0(j);
            if (column < P.D) to[column] = (lds[0][n] + lds[1][n]) + (lds[2][n] + lds[3][n]);
        }
}

__global__ void __launch_bounds__(1024) mrf_rotate_sum(const MrfRotateParams P)
{
    __shared__ float part[64][17];
    const int kind = blockIdx.y, w = threadIdx.x % 16, s = threadIdx.x / 16, column = blockIdx.x * 16 + w;
    if (!P.dgamma[kind] || P.blocks[kind] == 1) return;
    float v = 0.0f;
    if (column < P.D)
        for (int p = s; p < P.blocks[kind]; p += 64) v += P.partial[((size_t)kind * MRF_ROTATE_PARTS + p) * P.D + column];
    part[s][w] = v;
    __syncthreads();
    for (int d = 32; d > 0; d /= 2) {
        if (s < d) part[s][w] += part[s + d][w];
        __syncthreads();
    }
    if (s == 0 && column < P.D) P.dgamma[kind][column] = part[0][w];
}

namespace mrf_host {

template <bool FORWARD, class X, int S, int TL> static int rotate_go(const MrfRotateParams &P, bool whole, hipStream_t st)
{
    const unsigned grid = (unsigned)(P.blocks[0] + P.blocks[1]);
    if constexpr (FORWARD) {
        if (whole) mrf_rotate_fwd<X, S, TL, true><<<grid, 256, 0, st>>>(P);
        else mrf_rotate_fwd<X, S, TL, false><<<grid, 256, 0, st>>>(P);
        return launch_status("mrf_rotate_fwd");
    } else {
        if (whole) mrf_rotate_bwd<X, S, TL, true><<<grid, 256, 0, st>>>(P);
        else mrf_rotate_bwd<X, S, TL, false><<<grid, 256, 0, st>>>(P);
        if ((P.dgamma[0] && P.blocks[0] != 1) || (P.dgamma[1] && P.blocks[1] != 1)) mrf_rotate_sum<<<dim3((P.D + 15) / 16, 2), 1024, 0, st>>>(P);
        return launch_status("mrf_rotate_bwd");
    }
}

template <bool FORWARD, class X, int S> static int rotate_lanes(MrfRotateParams P, hipStream_t st)
{
    const int lanes = ((P.D + 1) / 2 + S - 1) / S, heads = P.Hq + P.Hk;
    int TL = 1;
    while (TL < lanes) TL *= 2;
    // heads a group: all of a token's where tokens alone keep the card busy (the angles are formed once), else fewer, down to one
    long long want = (131072 + P.tokens * TL - 1) / (P.tokens * TL);      // groups of a token for 512 workgroups
    if (want > heads) want = heads;
    P.heads = (int)((heads + want - 1) / want);
    if (P.heads > 4) P.heads -= P.heads % 4;
    const long long most = FORWARD ? 1 << 22 : MRF_ROTATE_PARTS;      // (a grid has fewer than 2^32 threads)
    for (int k = 0; k < 2; ++k) {
        P.pieces[k] = ((k ? P.Hk : P.Hq) + P.heads - 1) / P.heads;
        const long long blocks = (P.tokens * P.pieces[k] + 256 / TL - 1) / (256 / TL);
        P.blocks[k] = (int)(blocks < most ? blocks : most);
    }
    // runs of S neighbours: pairs that turn and the rest of a head in whole ones
    const bool whole = P.D % (2 * S) == 0 && (P.interleaved || P.half % S == 0);
    switch (TL) {
        case 1: return rotate_go<FORWARD, X, S, 1>(P, whole, st);
        case 2: return rotate_go<FORWARD, X, S, 2>(P, whole, st);
        case 4: return rotate_go<FORWARD, X, S, 4>(P, whole, st);
        case 8: return rotate_go<FORWARD, X, S, 8>(P, whole, st);
        case 16: return rotate_go<FORWARD, X, S, 16>(P, whole, st);
        case 32: return rotate_go<FORWARD, X, S, 32>(P, whole, st);
        default: return rotate_go<FORWARD, X, S, 64>(P, whole, st);
    }
}

// runs of 16 bytes where the head has whole ones, else of half of that in 16 bits
template <bool FORWARD, class X> static int rotate_typed(const MrfRotateParams &P, hipStream_t st)
{
    if constexpr (sizeof(X) == 2)
        if (P.D % 16 == 0 && (P.interleaved || P.half % 8 == 0)) return rotate_lanes<FORWARD, X, 8>(P, st);
    return rotate_lanes<FORWARD, X, 4>(P, st);
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
        if (none) {      // sums over nothing
            mrf_rotate_sum<<<dim3((P.D + 15) / 16, 2), 1024, 0, (hipStream_t)hip_stream>>>(P);
            return launch_status("mrf_rotate_sum");
        }
    }
    if (none) return MRF_OK;
    return rotate_launch<false>(P, heads->type, (hipStream_t)hip_stream);
}

}  // extern "C"
