// Gated linear recurrence along the middle index of [outer][T][inner], forward and backward (see mrf_gated_scan_forward in the header for the
// formulas).
//
// A lane has V neighbouring channels, MRF_SCAN_STEPS of their steps in registers.  The wavefronts of a workgroup have the same channels and the steps behind one another's:
// what a wavefront's steps do to the state they get is h -> A h + B; these meet in LDS, and each goes through its steps from the right state.  So every
// element is read once, and few channels still make many wavefronts.  Some 20 operations and two transcendental ones an element: bound by memory.
// Where there are too few channels for that, the steps are divided into chunks: a first launch finds what each does, a second one strings that
// together, and the third goes through the steps again.  The states before every MRF_SCAN_STEPS-th step are kept for the backward pass, in 32 bits:
// it forms the steps between them again in registers, whatever the type of y.  4 x 512 steps of 16,384 channels, 16 bits: forward 56 us (3.7 TB/s), backward 88 (3.9), in 32
// bits 222 together (4.8; a copy reaches 5.1); 65,537 steps of 256 channels, 32 bits, divided: forward 37 + 8 + 34, backward 25 + 8 + 67.  Four channels a lane in 16 bits
// took twice as long (333 us instead of 147: half the wavefronts, and registers in memory).
#include "mrfmp_rows.h"

#include <type_traits>

#define MRF_SCAN_STEPS 16
#define MRF_SCAN_WAVES 8      // of a workgroup, at most

struct MrfScanParams {
    long long outer, T, inner, groups, lanes;      // groups of V channels in a row of `inner`; lanes = outer groups
    const void *x, *z, *dy;
    long long x_outer, x_step, z_outer, z_step;    // elements from one row to the next
    const int *lengths;
    const float *start;                            // state before the first step (gradient behind the last): [outer][inner] or NULL
    void *y, *dx, *dz;
    float *end;                                    // state behind the last step (gradient before the first) or NULL
    float *states;                                 // [outer][blocks][inner]
    float2 *effect;                                // [chunks][outer inner]: A, B of a chunk
    float *carry;                                  // [chunks][outer inner]: state that a chunk gets
    long long chunk, blocks;
    int chunks;
};

// The logistic function of z and of -z.  The exponential is of a number below 0, so neither loses digits; NaN stays.
__device__ inline void mrf_gate(float z, float &a, float &rest)
{
    const float e = __builtin_amdgcn_exp2f(fabsf(z) * -1.44269504088896340736f);
    const float r = __builtin_amdgcn_rcpf(1.0f + e), low = e * r;
    a = z < 0.0f ? low : r;
    rest = z < 0.0f ? r : low;
}

template <class X, int V> struct MrfScanLane {
    typedef typename MrfVec<X, V>::type vec;
    typedef typename MrfVec<float, V>::type fvec;
    struct Raw { vec v[MRF_SCAN_STEPS]; };

    long long index, o;      // of outer * inner; row
    int n, i;                // steps that there are; first channel
    bool there;

    __device__ inline MrfScanLane(const MrfScanParams &P)
    {
        const long long lane = (long long)blockIdx.x * 64 + (threadIdx.x & 63);
        there = lane < P.lanes;
        o = there ? lane / P.groups : 0;
        i = (int)(lane - o * P.groups) * V;
        index = o * P.inner + i;
        n = (int)P.T;
        if (there && P.lengths) {
            n = P.lengths[o];
            n = n < 0 ? 0 : n > P.T ? (int)P.T : n;
        }
    }

    // steps u .. u + MRF_SCAN_STEPS - 1 of rows `step` apart from `row0` on (the row of step 0); nothing from `end` on
    __device__ inline void load(const X *row0, long long step, long long u, long long end, Raw &r) const
    {
        const X *at = row0 + u * step;
        if (u + MRF_SCAN_STEPS <= end) {
#pragma unroll
            for (int s = 0; s < MRF_SCAN_STEPS; ++s) r.v[s] = *(const vec *)(at + s * step);
        } else {
#pragma unroll
            for (int s = 0; s < MRF_SCAN_STEPS; ++s) {
                vec v;
#pragma unroll
                for (int j = 0; j < V; ++j) v[j] = (X)0.0f;
                if (u + s < end) v = *(const vec *)(at + s * step);
                r.v[s] = v;
            }
        }
    }

    static __device__ inline void state(const float *at, float (&h)[V])
    {
        const fvec v = *(const fvec *)at;
#pragma unroll
        for (int j = 0; j < V; ++j) h[j] = v[j];
    }
    static __device__ inline void keep(float *at, const float (&h)[V])
    {
        fvec v;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = h[j];
        *(fvec *)at = v;
    }
    static __device__ inline void give(X *at, const float (&h)[V])
    {
        vec v;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = mrf_from_f32<X>(h[j]);
        *(vec *)at = v;
    }
};

// rows of step 0 and the way from one step to the next
template <class X, bool REV> struct MrfScanRows {
    const X *row0;
    long long step;
    __device__ inline MrfScanRows(const void *base, long long outer, long long way, long long o, int n, int i)
    {
        row0 = (const X *)base + o * outer + i + (REV ? (long long)(n - 1) * way : 0);
        step = REV ? -way : way;
    }
};

// What the wavefronts of a workgroup do to a state, one behind the other
template <int V> struct MrfScanParts {
    float2 part[2][MRF_SCAN_WAVES][V][64];

    // h: the state before all wavefronts' steps, and then that behind them; returned in `mine`: the state before this one's, which do A, B to it
    __device__ inline void meet(int buf, int wv, int waves, const float (&A)[V], const float (&B)[V], float (&h)[V], float (&mine)[V])
    {
        const int lane = threadIdx.x & 63;
        if (waves == 1) {
#pragma unroll
            for (int j = 0; j < V; ++j) mine[j] = h[j], h[j] = fmaf(A[j], h[j], B[j]);
            return;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) part[buf][wv][j][lane] = make_float2(A[j], B[j]);
        __syncthreads();
        for (int w = 0; w < waves; ++w)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (w == wv) mine[j] = h[j];
                const float2 p = part[buf][w][j][lane];
                h[j] = fmaf(p.x, h[j], p.y);
            }
    }

    // h, all: what is done to a state so far (all h0 + h), and then by all wavefronts' steps too
    __device__ inline void pass(int buf, int wv, int waves, const float (&A)[V], const float (&B)[V], float (&h)[V], float (&all)[V])
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < V; ++j) part[buf][wv][j][lane] = make_float2(A[j], B[j]);
        __syncthreads();
        for (int w = 0; w < waves; ++w)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float2 p = part[buf][w][j][lane];
                h[j] = fmaf(p.x, h[j], p.y);
                all[j] *= p.x;
            }
    }
};

template <class X, int V, bool COMPLEMENT, bool REV>
__global__ void __launch_bounds__(64 * MRF_SCAN_WAVES) mrf_scan_fwd(const MrfScanParams P)
{
    typedef MrfScanLane<X, V> Lane;
    __shared__ MrfScanParts<V> parts;
    const Lane me(P);
    const int wv = threadIdx.x >> 6, waves = blockDim.x >> 6, ahead = waves * MRF_SCAN_STEPS;
    const long long from = (long long)blockIdx.y * P.chunk, to = from + P.chunk < P.T ? from + P.chunk : P.T;
    const long long last = !me.there ? 0 : me.n < to ? me.n : to;
    float h[V];
#pragma unroll
    for (int j = 0; j < V; ++j) h[j] = 0.0f;
    if (me.there) {
        if (P.chunks > 1) Lane::state(P.carry + blockIdx.y * (P.outer * P.inner) + me.index, h);
        else if (P.start) Lane::state(P.start + me.index, h);
    }
    const MrfScanRows<X, REV> x(P.x, P.x_outer, P.x_step, me.o, me.n, me.i), z(P.z, P.z_outer, P.z_step, me.o, me.n, me.i);
    const long long dense = P.T * P.inner;
    X *const y = (X *)P.y + me.o * dense + me.i;
    int buf = 0;

    const auto run = [&](const typename Lane::Raw &rx, const typename Lane::Raw &rz, const long long u) {
        float a[MRF_SCAN_STEPS][V], b[MRF_SCAN_STEPS][V], A[V], B[V], mine[V];
#pragma unroll
        for (int j = 0; j < V; ++j) A[j] = 1.0f, B[j] = 0.0f;
#pragma unroll
        for (int s = 0; s < MRF_SCAN_STEPS; ++s)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float rest;
                mrf_gate(mrf_to_f32((X)rz.v[s][j]), a[s][j], rest);
                const float v = mrf_to_f32((X)rx.v[s][j]);
                b[s][j] = COMPLEMENT ? rest * v : v;
                if (u + s >= last) a[s][j] = 1.0f, b[s][j] = 0.0f;
                B[j] = fmaf(a[s][j], B[j], b[s][j]);
                A[j] *= a[s][j];
            }
        parts.meet(buf, wv, waves, A, B, h, mine);
        buf ^= 1;
        if (!me.there) return;
        if (P.states && u < to) Lane::keep(P.states + (me.o * P.blocks + u / MRF_SCAN_STEPS) * P.inner + me.i, mine);
#pragma unroll
        for (int s = 0; s < MRF_SCAN_STEPS; ++s) {
            if (u + s < last) {
#pragma unroll
                for (int j = 0; j < V; ++j) mine[j] = fmaf(a[s][j], mine[j], b[s][j]);
                Lane::give(y + (REV ? me.n - 1 - (u + s) : u + s) * P.inner, mine);
            } else if (u + s < to) {
                const float zero[V] = {};
                Lane::give(y + (u + s) * P.inner, zero);
            }
        }
        if (waves == 1) {      // (as the steps round it)
#pragma unroll
            for (int j = 0; j < V; ++j) h[j] = mine[j];
        }
    };
    typename Lane::Raw xa, za, xb, zb;
    const auto load = [&](long long u, typename Lane::Raw &rx, typename Lane::Raw &rz) {
        me.load(x.row0, x.step, u, last, rx);
        me.load(z.row0, z.step, u, last, rz);
    };
    // (`first` is the same in all threads)
    if (from < to) load(from + wv * MRF_SCAN_STEPS, xa, za);
    for (long long first = from; first < to; first += 2 * ahead) {
        const long long u = first + wv * MRF_SCAN_STEPS;
        const bool more = first + ahead < to;
        if (more) load(u + ahead, xb, zb);
        run(xa, za, u);
        if (first + 2 * ahead < to) load(u + 2 * ahead, xa, za);
        if (more) run(xb, zb, u + ahead);
    }
    if (blockIdx.y == (unsigned)P.chunks - 1 && P.end && wv == 0 && me.there) Lane::keep(P.end + me.index, h);
}

// What a chunk does to the state it gets: h -> A h + B
template <class X, int V, bool COMPLEMENT, bool REV> __global__ void __launch_bounds__(64 * MRF_SCAN_WAVES) mrf_scan_fwd_effect(const MrfScanParams P)
{
    typedef MrfScanLane<X, V> Lane;
    __shared__ MrfScanParts<V> parts;
    const Lane me(P);
    const int wv = threadIdx.x >> 6, waves = blockDim.x >> 6, ahead = waves * MRF_SCAN_STEPS;
    const long long from = (long long)blockIdx.y * P.chunk, to = from + P.chunk < P.T ? from + P.chunk : P.T;
    const long long last = !me.there ? 0 : me.n < to ? me.n : to;
    float all[V], h[V];
#pragma unroll
    for (int j = 0; j < V; ++j) all[j] = 1.0f, h[j] = 0.0f;
    const MrfScanRows<X, REV> x(P.x, P.x_outer, P.x_step, me.o, me.n, me.i), z(P.z, P.z_outer, P.z_step, me.o, me.n, me.i);
    int buf = 0;
    for (long long first = from; first < to; first += ahead, buf ^= 1) {
        const long long u = first + wv * MRF_SCAN_STEPS;
        typename Lane::Raw rx, rz;
        float A[V], B[V];
        me.load(z.row0, z.step, u, last, rz);
        me.load(x.row0, x.step, u, last, rx);
#pragma unroll
        for (int j = 0; j < V; ++j) A[j] = 1.0f, B[j] = 0.0f;
#pragma unroll
        for (int s = 0; s < MRF_SCAN_STEPS; ++s)
            if (u + s < last) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float a, rest;
                    mrf_gate(mrf_to_f32((X)rz.v[s][j]), a, rest);
                    const float v = mrf_to_f32((X)rx.v[s][j]);
                    B[j] = fmaf(a, B[j], COMPLEMENT ? rest * v : v);
                    A[j] *= a;
                }
            }
        parts.pass(buf, wv, waves, A, B, h, all);
    }
    if (me.there && wv == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) P.effect[blockIdx.y * (P.outer * P.inner) + me.index + j] = make_float2(all[j], h[j]);
    }
}

// Backward: c is what reaches a step's state from the steps behind it; g = dy + c, and the step before gets a g.  The wavefronts have the steps in front of one
// another's: what a wavefront's steps do to c is c -> A c + B.
template <class X, int V, bool COMPLEMENT, bool REV>
__global__ void __launch_bounds__(64 * MRF_SCAN_WAVES) mrf_scan_bwd(const MrfScanParams P)
{
    typedef MrfScanLane<X, V> Lane;
    __shared__ MrfScanParts<V> parts;
    const Lane me(P);
    const int wv = threadIdx.x >> 6, waves = blockDim.x >> 6, ahead = waves * MRF_SCAN_STEPS;
    const long long from = (long long)blockIdx.y * P.chunk, to = from + P.chunk < P.T ? from + P.chunk : P.T;
    const long long last = !me.there ? 0 : me.n < to ? me.n : to;
    float c[V];
#pragma unroll
    for (int j = 0; j < V; ++j) c[j] = 0.0f;
    if (me.there) {
        if (P.chunks > 1) Lane::state(P.carry + blockIdx.y * (P.outer * P.inner) + me.index, c);
        else if (P.start) Lane::state(P.start + me.index, c);
    }
    const MrfScanRows<X, REV> x(P.x, P.x_outer, P.x_step, me.o, me.n, me.i), z(P.z, P.z_outer, P.z_step, me.o, me.n, me.i);
    const long long dense = P.T * P.inner;
    const MrfScanRows<X, REV> dy(P.dy, dense, P.inner, me.o, me.n, me.i);
    X *const dx = (X *)P.dx + me.o * dense + me.i, *const dz = (X *)P.dz + me.o * dense + me.i;
    int buf = 0;

    // (`top` is the same in all threads)
    for (long long top = to > from ? (to - 1) / MRF_SCAN_STEPS * MRF_SCAN_STEPS : from - 1; top >= from; top -= ahead) {
        const long long u = top - wv * MRF_SCAN_STEPS;      // (below `from` there is nothing for this wavefront)
        const bool steps = u >= from && u < last;
        typename Lane::Raw rx, rz, ry;
        float h[V], before[MRF_SCAN_STEPS][V], a[MRF_SCAN_STEPS][V], rest[MRF_SCAN_STEPS][V], A[V], B[V], mine[V];
#pragma unroll
        for (int j = 0; j < V; ++j) A[j] = 1.0f, B[j] = 0.0f;
        if (steps) {
            me.load(z.row0, z.step, u, last, rz);
            me.load(dy.row0, dy.step, u, last, ry);
            me.load(x.row0, x.step, u, last, rx);
            Lane::state(P.states + (me.o * P.blocks + u / MRF_SCAN_STEPS) * P.inner + me.i, h);
#pragma unroll
            for (int s = MRF_SCAN_STEPS - 1; s >= 0; --s)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    mrf_gate(mrf_to_f32((X)rz.v[s][j]), a[s][j], rest[s][j]);
                    if (u + s < last) {
                        B[j] = a[s][j] * (mrf_to_f32((X)ry.v[s][j]) + B[j]);
                        A[j] *= a[s][j];
                    }
                }
#pragma unroll
            for (int s = 0; s < MRF_SCAN_STEPS; ++s)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const float v = mrf_to_f32((X)rx.v[s][j]);
                    before[s][j] = h[j];
                    h[j] = fmaf(a[s][j], h[j], COMPLEMENT ? rest[s][j] * v : v);
                }
        }
        parts.meet(buf, wv, waves, A, B, c, mine);
        buf ^= 1;
        if (steps) {
#pragma unroll
            for (int s = MRF_SCAN_STEPS - 1; s >= 0; --s) {
                if (u + s < last) {
                    float gx[V], gz[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float g = mrf_to_f32((X)ry.v[s][j]) + mine[j], ag = a[s][j] * g;
                        gx[j] = COMPLEMENT ? rest[s][j] * g : g;
                        gz[j] = ag * rest[s][j] * (COMPLEMENT ? before[s][j] - mrf_to_f32((X)rx.v[s][j]) : before[s][j]);
                        mine[j] = ag;
                    }
                    const long long t = REV ? me.n - 1 - (u + s) : u + s;
                    if (P.dx) Lane::give(dx + t * P.inner, gx);
                    if (P.dz) Lane::give(dz + t * P.inner, gz);
                }
            }
        }
        if (me.there && u >= from && u + MRF_SCAN_STEPS > last) {
            const float zero[V] = {};
            for (int s = 0; s < MRF_SCAN_STEPS; ++s)
                if (u + s >= last && u + s < to) {
                    if (P.dx) Lane::give(dx + (u + s) * P.inner, zero);
                    if (P.dz) Lane::give(dz + (u + s) * P.inner, zero);
                }
        }
        if (waves == 1 && steps) {
#pragma unroll
            for (int j = 0; j < V; ++j) c[j] = mine[j];
        }
    }
    if (blockIdx.y == 0 && P.end && wv == 0 && me.there) Lane::keep(P.end + me.index, c);
}

// What a chunk does to the gradient that reaches it from behind: c -> A c + B
template <class X, int V, bool REV> __global__ void __launch_bounds__(64 * MRF_SCAN_WAVES) mrf_scan_bwd_effect(const MrfScanParams P)
{
    typedef MrfScanLane<X, V> Lane;
    __shared__ MrfScanParts<V> parts;
    const Lane me(P);
    const int wv = threadIdx.x >> 6, waves = blockDim.x >> 6, ahead = waves * MRF_SCAN_STEPS;
    const long long from = (long long)blockIdx.y * P.chunk, to = from + P.chunk < P.T ? from + P.chunk : P.T;
    const long long last = !me.there ? 0 : me.n < to ? me.n : to;
    float all[V], c[V];
#pragma unroll
    for (int j = 0; j < V; ++j) all[j] = 1.0f, c[j] = 0.0f;
    const MrfScanRows<X, REV> z(P.z, P.z_outer, P.z_step, me.o, me.n, me.i);
    const MrfScanRows<X, REV> dy(P.dy, P.T * P.inner, P.inner, me.o, me.n, me.i);
    int buf = 0;
    for (long long top = to > from ? (to - 1) / MRF_SCAN_STEPS * MRF_SCAN_STEPS : from - 1; top >= from; top -= ahead, buf ^= 1) {
        const long long u = top - wv * MRF_SCAN_STEPS;
        typename Lane::Raw rz, ry;
        float A[V], B[V];
#pragma unroll
        for (int j = 0; j < V; ++j) A[j] = 1.0f, B[j] = 0.0f;
        if (u >= from) {
            me.load(z.row0, z.step, u, last, rz);
            me.load(dy.row0, dy.step, u, last, ry);
#pragma unroll
            for (int s = MRF_SCAN_STEPS - 1; s >= 0; --s)
                if (u + s < last) {
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        float a, rest;
                        mrf_gate(mrf_to_f32((X)rz.v[s][j]), a, rest);
                        B[j] = a * (mrf_to_f32((X)ry.v[s][j]) + B[j]);
                        A[j] *= a;
                    }
                }
        }
        parts.pass(buf, wv, waves, A, B, c, all);
    }
    if (me.there && wv == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) P.effect[blockIdx.y * (P.outer * P.inner) + me.index + j] = make_float2(all[j], c[j]);
    }
}

// States that the chunks get, from what each does to them, in the order of the chunks (backward: from the last).  A workgroup has 16 channels, 64 threads
// for each of them with as many chunks in a row; what those do together meets in LDS.
template <bool BACK>
__global__ void __launch_bounds__(1024) mrf_scan_carry(const MrfScanParams P)
{
    __shared__ float2 part[64][16];
    const int w = threadIdx.x % 16, s = threadIdx.x / 16;
    const long long N = P.outer * P.inner, i = (long long)blockIdx.x * 16 + w;
    const int per = (P.chunks + 63) / 64, p0 = s * per < P.chunks ? s * per : P.chunks, p1 = p0 + per < P.chunks ? p0 + per : P.chunks;
    const auto at = [&](int p) { return (size_t)(BACK ? P.chunks - 1 - p : p) * N + i; };
    float A = 1.0f, B = 0.0f;
    if (i < N)
        for (int p = p0; p < p1; ++p) {
            const float2 e = P.effect[at(p)];
            B = fmaf(e.x, B, e.y);
            A *= e.x;
        }
    part[s][w] = make_float2(A, B);
    __syncthreads();
    for (int d = 1; d < 64; d *= 2) {
        const float2 mine = part[s][w], other = s >= d ? part[s - d][w] : make_float2(1.0f, 0.0f);
        __syncthreads();
        part[s][w] = make_float2(mine.x * other.x, fmaf(mine.x, other.y, mine.y));
        __syncthreads();
    }
    if (i >= N) return;
    float h = P.start ? P.start[i] : 0.0f;
    if (s > 0) h = fmaf(part[s - 1][w].x, h, part[s - 1][w].y);
    for (int p = p0; p < p1; ++p) {
        P.carry[at(p)] = h;
        const float2 e = P.effect[at(p)];
        h = fmaf(e.x, h, e.y);
    }
}

// A single step, forward and backward: a lane has V channels, and nothing is prepared for more: a million channels take 17 us forward
// and backward together, and took 50 with the kernels above.
template <class X, int V, bool COMPLEMENT, bool BACK> __global__ void __launch_bounds__(256) mrf_scan_one(const MrfScanParams P)
{
    typedef MrfScanLane<X, V> Lane;
    typedef typename Lane::vec vec;
    const long long lane = (long long)blockIdx.x * 256 + threadIdx.x;
    if (lane >= P.lanes) return;
    const long long o = lane / P.groups;
    const int i = (int)(lane - o * P.groups) * V;
    const long long index = o * P.inner + i;
    const bool there = !P.lengths || P.lengths[o] > 0;
    float h[V] = {}, a[V], rest[V], v[V], y[V] = {}, z[V] = {};
    if (there) {
        const vec x = *(const vec *)((const X *)P.x + o * P.x_outer + i), g = *(const vec *)((const X *)P.z + o * P.z_outer + i);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            v[j] = mrf_to_f32((X)x[j]);
            mrf_gate(mrf_to_f32((X)g[j]), a[j], rest[j]);
        }
    }
    if constexpr (!BACK) {
        if (P.start) Lane::state(P.start + index, h);
        if (P.states) Lane::keep(P.states + index, h);
        if (there) {
#pragma unroll
            for (int j = 0; j < V; ++j) y[j] = h[j] = fmaf(a[j], h[j], COMPLEMENT ? rest[j] * v[j] : v[j]);
        }
        Lane::give((X *)P.y + index, y);
        if (P.end) Lane::keep(P.end + index, h);
    } else {
        float c[V] = {};
        if (P.start) Lane::state(P.start + index, c);
        if (there) {
            Lane::state(P.states + index, h);
            const vec dy = *(const vec *)((const X *)P.dy + index);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float g = mrf_to_f32((X)dy[j]) + c[j], ag = a[j] * g;
                y[j] = COMPLEMENT ? rest[j] * g : g;
                z[j] = ag * rest[j] * (COMPLEMENT ? h[j] - v[j] : h[j]);
                c[j] = ag;
            }
        }
        if (P.dx) Lane::give((X *)P.dx + index, y);
        if (P.dz) Lane::give((X *)P.dz + index, z);
        if (P.end) Lane::keep(P.end + index, c);
    }
}

namespace mrf_host {

struct ScanSplit { int chunks; long long chunk; };

// Chunks of the steps: none where a workgroup's wavefronts make enough of the channels alone.
static ScanSplit scan_split(long long outer, long long T, long long inner)
{
    const long long N = outer * inner;
    if (N >= 8192 || T <= 1024 || N == 0) return {1, T};
    long long P = (262144 + N - 1) / N;
    if (P > (T + 127) / 128) P = (T + 127) / 128;
    if (P > 16384) P = 16384;
    const long long chunk = ((T + P - 1) / P + MRF_SCAN_STEPS - 1) / MRF_SCAN_STEPS * MRF_SCAN_STEPS;
    return {(int)((T + chunk - 1) / chunk), chunk};
}

static bool scan_sizes_ok(long long outer, long long T, long long inner)
{
    const long long most = 0x7fffffffLL;
    if (outer < 0 || T < 0 || inner < 0 || outer > most || T > most - 2 * MRF_SCAN_STEPS || inner > most) return false;
    if (outer && inner > most / outer) return false;      // (channels: a grid has fewer than 2^32 threads)
    return !(outer && inner && T) || T <= (1LL << 60) / (outer * inner);
}

// Wavefronts of a workgroup: as many as make 4,096 of them, as far as a chunk has steps for them.
static unsigned scan_waves(const MrfScanParams &P)
{
    const long long groups = (P.lanes + 63) / 64 * P.chunks;
    int waves = 1;
    while (waves < MRF_SCAN_WAVES && groups * waves < 4096 && waves * MRF_SCAN_STEPS < P.chunk) waves *= 2;
    return 64 * waves;
}

template <class X, int V, bool REV> static int scan_forward(MrfScanParams P, bool complement, hipStream_t st)
{
    P.groups = P.inner / V;
    P.lanes = P.outer * P.groups;
    if (P.T == 1) {
        const unsigned blocks = (unsigned)((P.lanes + 255) / 256);
        if (complement) mrf_scan_one<X, V, true, false><<<blocks, 256, 0, st>>>(P);
        else mrf_scan_one<X, V, false, false><<<blocks, 256, 0, st>>>(P);
        return launch_status("mrf_scan_one");
    }
    const unsigned threads = scan_waves(P);
    const dim3 grid((unsigned)((P.lanes + 63) / 64), (unsigned)P.chunks);
    if (P.chunks > 1) {
        if (complement) mrf_scan_fwd_effect<X, V, true, REV><<<grid, threads, 0, st>>>(P);
        else mrf_scan_fwd_effect<X, V, false, REV><<<grid, threads, 0, st>>>(P);
        mrf_scan_carry<false><<<(unsigned)((P.outer * P.inner + 15) / 16), 1024, 0, st>>>(P);
    }
    if (complement) mrf_scan_fwd<X, V, true, REV><<<grid, threads, 0, st>>>(P);
    else mrf_scan_fwd<X, V, false, REV><<<grid, threads, 0, st>>>(P);
    return launch_status("mrf_scan_fwd");
}

template <class X, int V, bool REV> static int scan_backward(MrfScanParams P, bool complement, hipStream_t st)
{
    P.groups = P.inner / V;
    P.lanes = P.outer * P.groups;
    if (P.T == 1) {
        const unsigned blocks = (unsigned)((P.lanes + 255) / 256);
        if (complement) mrf_scan_one<X, V, true, true><<<blocks, 256, 0, st>>>(P);
        else mrf_scan_one<X, V, false, true><<<blocks, 256, 0, st>>>(P);
        return launch_status("mrf_scan_one");
    }
    const unsigned threads = scan_waves(P);
    const dim3 grid((unsigned)((P.lanes + 63) / 64), (unsigned)P.chunks);
    if (P.chunks > 1) {
        mrf_scan_bwd_effect<X, V, REV><<<grid, threads, 0, st>>>(P);
        mrf_scan_carry<true><<<(unsigned)((P.outer * P.inner + 15) / 16), 1024, 0, st>>>(P);
    }
    if (complement) mrf_scan_bwd<X, V, true, REV><<<grid, threads, 0, st>>>(P);
    else mrf_scan_bwd<X, V, false, REV><<<grid, threads, 0, st>>>(P);
    return launch_status("mrf_scan_bwd");
}

// two channels a lane where 16 bits and an even row allow it (a load of 4 bytes), unless that leaves too few workgroups
template <bool FORWARD> static int scan_launch(const MrfScanParams &P, int type, bool complement, bool reverse, hipStream_t st)
{
    const auto go = [&](auto x, auto v, auto rev) {
        typedef decltype(x) X;
        if constexpr (FORWARD) return scan_forward<X, decltype(v)::value, decltype(rev)::value>(P, complement, st);
        else return scan_backward<X, decltype(v)::value, decltype(rev)::value>(P, complement, st);
    };
    const auto typed = [&](auto x) {
        if constexpr (sizeof(x) == 2)
            if (P.inner % 2 == 0 && (P.chunks > 1 || P.outer * P.inner >= 32768))
                return reverse ? go(x, std::integral_constant<int, 2>{}, std::true_type{}) : go(x, std::integral_constant<int, 2>{}, std::false_type{});
        return reverse ? go(x, std::integral_constant<int, 1>{}, std::true_type{}) : go(x, std::integral_constant<int, 1>{}, std::false_type{});
    };
    if (type == MRF_F32) return typed(0.0f);
    return type == MRF_F16 ? typed((mrf_f16)0.0f) : typed((mrf_bf16)0.0f);
}

static size_t scan_workspace(long long outer, long long T, long long inner)
{
    const ScanSplit s = scan_split(outer, T, inner);
    return s.chunks > 1 ? (size_t)s.chunks * outer * inner * 12 : 0;
}

static int scan_prepare(MrfScanParams &P, int type, void *workspace, size_t workspace_bytes)
{
    const ScanSplit s = scan_split(P.outer, P.T, P.inner);
    P.chunks = s.chunks;
    P.chunk = s.chunk;
    P.blocks = (P.T + MRF_SCAN_STEPS - 1) / MRF_SCAN_STEPS;
    if (!known_type(type) || P.x_outer < 0 || P.x_step < 0 || P.z_outer < 0 || P.z_step < 0) return MRF_ERR_BAD_ARGUMENT;
    if (P.outer == 0 || P.inner == 0) return MRF_OK;
    if (P.T > 0 && (!P.x || !P.z)) return MRF_ERR_NULL_POINTER;
    if (s.chunks > 1) {
        if (!workspace) return MRF_ERR_NULL_POINTER;
        if (workspace_bytes < scan_workspace(P.outer, P.T, P.inner)) return MRF_ERR_WORKSPACE_TOO_SMALL;
        P.effect = (float2 *)workspace;
        P.carry = (float *)(P.effect + (size_t)s.chunks * P.outer * P.inner);
    }
    return MRF_OK;
}

}  // namespace mrf_host

using namespace mrf_host;

extern "C" {

int64_t mrf_gated_scan_states(int64_t T) { return T < 0 ? 0 : (T + MRF_SCAN_STEPS - 1) / MRF_SCAN_STEPS; }

size_t mrf_gated_scan_workspace_bytes(int64_t n_outer, int64_t T, int64_t n_inner)
{
    return scan_sizes_ok(n_outer, T, n_inner) ? scan_workspace(n_outer, T, n_inner) : 0;
}

int mrf_gated_scan_forward(int64_t n_outer, int64_t T, int64_t n_inner, int type, const void *x, const int64_t *x_strides, const void *z,
                           const int64_t *z_strides, int complement, int reverse, const float *initial, const int32_t *lengths, void *y,
                           float *final_state, float *states, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!scan_sizes_ok(n_outer, T, n_inner)) return MRF_ERR_BAD_SHAPE;
    MrfScanParams P = {};
    P.outer = n_outer; P.T = T; P.inner = n_inner; P.x = x; P.z = z; P.lengths = lengths; P.start = initial; P.y = y; P.end = final_state;
    P.states = states;
    P.x_outer = x_strides ? x_strides[0] : T * n_inner; P.x_step = x_strides ? x_strides[1] : n_inner;
    P.z_outer = z_strides ? z_strides[0] : T * n_inner; P.z_step = z_strides ? z_strides[1] : n_inner;
    const int rc = scan_prepare(P, type, workspace, workspace_bytes);
    if (rc != MRF_OK || n_outer == 0 || n_inner == 0) return rc;
    if (T > 0 && !y) return MRF_ERR_NULL_POINTER;
    return scan_launch<true>(P, type, complement != 0, reverse != 0, (hipStream_t)hip_stream);
}

int mrf_gated_scan_backward(int64_t n_outer, int64_t T, int64_t n_inner, int type, const void *grad_y, const float *grad_final, const void *x,
                            const int64_t *x_strides, const void *z, const int64_t *z_strides, int complement, int reverse,
                            const int32_t *lengths, const float *states, void *grad_x, void *grad_z, float *grad_initial, void *workspace,
                            size_t workspace_bytes, void *hip_stream)
{
    if (!scan_sizes_ok(n_outer, T, n_inner)) return MRF_ERR_BAD_SHAPE;
    MrfScanParams P = {};
    P.outer = n_outer; P.T = T; P.inner = n_inner; P.x = x; P.z = z; P.dy = grad_y; P.lengths = lengths; P.start = grad_final; P.dx = grad_x;
    P.dz = grad_z; P.end = grad_initial; P.states = (float *)states;
    P.x_outer = x_strides ? x_strides[0] : T * n_inner; P.x_step = x_strides ? x_strides[1] : n_inner;
    P.z_outer = z_strides ? z_strides[0] : T * n_inner; P.z_step = z_strides ? z_strides[1] : n_inner;
    const int rc = scan_prepare(P, type, workspace, workspace_bytes);
    if (rc != MRF_OK || n_outer == 0 || n_inner == 0) return rc;
    if (T > 0 && (!grad_y || !states)) return MRF_ERR_NULL_POINTER;
    return scan_launch<false>(P, type, complement != 0, reverse != 0, (hipStream_t)hip_stream);
}

}  // extern "C"
