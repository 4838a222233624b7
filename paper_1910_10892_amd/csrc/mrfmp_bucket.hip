// Pairwise functions from a table of label distances in buckets, and the table's gradient (see
// mrf_bucket_pairwise_forward in the header for the formulas).
#include "mrfmp_rows.h"

#include <type_traits>

struct MrfBucketParams {
    long long G;
    int Q, K, NB;
    const float *table;
    long long sg, sb;            // strides of the table: group, bucket
    const int *bucket_of;        // [Q + K - 1] buckets of the offsets from -(Q - 1) - query_offset on
    void *out;                   // forward [G][Q][K]
    const void *dout;            // backward
    float *dtable;
    float *totals;               // [G][Q + K - 1] sums along whole diagonals (long matrices)
    float *diagonals;            // [G][T][strips][..] sums along diagonals over a strip's columns and a part's rows (long matrices)
    int quads;                   // forward, many small matrices: fours of groups whose tables are in LDS at once
    int KL, TR;                  // forward, long matrices: lanes of a row, rows of a lane
    int groups, tile;            // backward, many small matrices: matrices of a wavefront, bytes of LDS for them
    int T, TQ, strips;           // backward, long matrices: parts of the rows, rows of a wavefront, strips of the columns
};

__device__ inline int mrf_bucket_clamped(int b, int NB) { return b < 0 ? 0 : (b < NB ? b : NB - 1); }

// ---- forward, many small matrices (Q K <= 4096).  Four matrices are Q K chunks of four entries, whatever Q and K: a thread keeps the places in
// the tables of the four entries of its chunks, in registers, and goes from four matrices to the next.  Chunks of neighbouring threads
// are neighbours in memory, and no index is computed twice.  Bound by what it writes: 262,144 matrices of 21 x 21 in 32 bits 85 to 90 us in a trace
// of single passes (5.3 TB/s and more, tables included), 92 to 103 where calls follow each other at once.
constexpr int MRF_BUCKET_SMALL = 4096, MRF_BUCKET_LDS = 4096, MRF_BUCKET_CHUNKS = 4;      // entries of a matrix; floats in LDS; chunks of a thread

template <class T, int NT>
__global__ void __launch_bounds__(NT) mrf_bucket_fwd_small(const MrfBucketParams P)
{
    typedef typename MrfVec<T, 4>::type vec;
    __shared__ float tables[MRF_BUCKET_LDS];
    const int S = P.Q * P.K, NB = P.NB, groups = 4 * P.quads;
    int at[MRF_BUCKET_CHUNKS][4];
#pragma unroll
    for (int c = 0; c < MRF_BUCKET_CHUNKS; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 4 * (int)(threadIdx.x + NT * c) + j;
            at[c][j] = 0;
            if (e < 4 * S) {
                const int g = e / S, r = e - g * S, q = r / P.K;
                at[c][j] = g * NB + mrf_bucket_clamped(P.bucket_of[r - q * P.K - q + (P.Q - 1)], NB);
            }
        }
    for (long long g0 = (long long)blockIdx.x * groups; g0 < P.G; g0 += (long long)gridDim.x * groups) {
        const int here = P.G - g0 < groups ? (int)(P.G - g0) : groups;
        if (P.sb == 1) {
            for (int i = threadIdx.x; i < here * NB; i += NT) tables[i] = P.table[g0 * NB + i];
        } else {
            for (int i = threadIdx.x; i < groups * NB; i += NT) {
                const int b = i / groups, g = i - b * groups;
                if (g < here) tables[g * NB + b] = P.table[b * P.sb + g0 + g];
            }
        }
        __syncthreads();
        T *out = (T *)P.out + (size_t)g0 * S;
        for (int f = 0; f < here; f += 4, out += 4 * (size_t)S) {
            const float *t = tables + f * NB;
            if (f + 4 <= here) {
#pragma unroll
                for (int c = 0; c < MRF_BUCKET_CHUNKS; ++c) {
                    const unsigned k = threadIdx.x + NT * c;
                    if (k < (unsigned)S) {
                        vec v;
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = mrf_from_f32<T>(t[at[c][j]]);
                        *(vec *)(out + 4 * k) = v;
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < MRF_BUCKET_CHUNKS; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int e = 4 * (int)(threadIdx.x + NT * c) + j;
                        if (e < (here - f) * S) out[e] = mrf_from_f32<T>(t[at[c][j]]);
                    }
            }
        }
        __syncthreads();
    }
}

// ---- forward, long matrices.  A row is the row above it moved by one: a wavefront lays the values along KL V columns and its rows out as one line
// in LDS, and a lane that goes down V columns reads one new value a row.  KL lanes share a row, 64 / KL runs of TR rows a wavefront.  Bound by what
// it writes: 16 matrices of 2,048 x 2,048 in 16 bits 29 us (4.7 TB/s); by the launch: 16 rows of 4,099 in 32 bits 4 us.
constexpr int MRF_BUCKET_RUNS = 256;      // rows of a wavefront at most

template <class T, int V>
__global__ void __launch_bounds__(256) mrf_bucket_fwd_long(const MrfBucketParams P)
{
    typedef MrfRow<1, V, 1> Piece;
    __shared__ float lines[4][64 * V + MRF_BUCKET_RUNS];
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int KL = P.KL, TR = P.TR, l = lane & (KL - 1), run = lane / KL, TQ = TR * (64 / KL), W = KL * V;
    const unsigned across = (unsigned)((P.K + W - 1) / W), down = (unsigned)((P.Q + TQ - 1) / TQ);
    const unsigned tile = blockIdx.x * 4u + (unsigned)wv;
    if (tile >= across * down) return;
    const int q0 = (int)(tile / across) * TQ, k0 = (int)(tile % across) * W;
    float *line = lines[wv];
    const int n = W + TQ - 1, first = k0 - (q0 + TQ - 1) + (P.Q - 1), last = P.Q + P.K - 2;
    const int q = q0 + run * TR, rows = P.Q - q < TR ? P.Q - q : TR, k = k0 + l * V, here = P.K - k;
    for (long long g = blockIdx.y; g < P.G; g += gridDim.y) {
        for (int i = lane; i < n; i += 64) {
            // (offsets that no entry has are left out)
            const int d = first + i;
            line[i] = d >= 0 && d <= last ? P.table[g * P.sg + mrf_bucket_clamped(P.bucket_of[d], P.NB) * P.sb] : 0.0f;
        }
        mrf_wave_lds_fence();
        T *out = (T *)P.out + ((size_t)g * P.Q + q) * P.K + k;
        const float *from = line + (l * V + (TQ - 1) - run * TR);
        float v[2 * V - 1];      // the entries of V rows: row i of them has v[V - 1 - i ...]
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = from[j];
        if (here > 0)
            for (int r = 0; r < rows; r += V) {
#pragma unroll
                for (int j = V - 1; j >= 0; --j) v[V - 1 + j] = v[j];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    if (i > 0) v[V - 1 - i] = r + i < rows ? from[-(r + i)] : 0.0f;
                    if (r + i < rows) {
                        float w[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) w[j] = v[V - 1 - i + j];
                        Piece::store(out + (size_t)(r + i) * P.K, here < V ? here : V, 0, w);
                    }
                }
                if (r + V < rows) {
                    // the next V rows begin one further up the line
#pragma unroll
                    for (int j = V - 1; j > 0; --j) v[j] = v[j - 1];
                    v[0] = from[-(r + V)];
                }
            }
        mrf_wave_lds_fence();
    }
}

// ---- backward.  A diagonal has one bucket: sums go down the diagonals first, where the lanes of a wavefront, one diagonal each, read neighbours in
// every row, and then over the diagonals of a bucket.

// Many small matrices (Q, K <= 64): a wavefront takes as many as have room in its lanes, neighbours in memory, into LDS as whole chunks.  Lanes
// j < K of a matrix go down its rows from column j on and begin again at column 0, so that none idles; where a lane begins again, a
// diagonal's sum is complete.  Bound by memory: 262,144 matrices of 21 x 21 in 32 bits 96 to 100 us (4.7 to 5.0 TB/s; right behind a forward call 147 to 152, which includes that call's
// writes on their way from the caches).
constexpr int MRF_BUCKET_SIDE = 64, MRF_BUCKET_DIAG = 512, MRF_BUCKET_MANY = 512, MRF_BUCKET_WAVES = 2;      // Q, K; diagonals of a wavefront; buckets; wavefronts

// NQ: chunks of a lane; the next matrices' are on their way while these are summed.
template <class T, bool WIDE, int NQ>
__global__ void __launch_bounds__(64 * MRF_BUCKET_WAVES) mrf_bucket_bwd_small(const MrfBucketParams P)
{
    typedef typename MrfChunk<sizeof(T)>::type chunk;
    typedef typename MrfChunk<16>::type quad;
    constexpr int NT = 64 * MRF_BUCKET_WAVES, PER = 16 / (int)sizeof(T);
    extern __shared__ __align__(16) char staged[];      // [MRF_BUCKET_WAVES][P.tile] bytes
    __shared__ float diag[MRF_BUCKET_WAVES][MRF_BUCKET_DIAG];
    __shared__ int bucket[2 * MRF_BUCKET_SIDE], place[2 * MRF_BUCKET_SIDE], begin[MRF_BUCKET_MANY + 1];
    const int Q = P.Q, K = P.K, NB = P.NB, S = Q * K, D = Q + K - 1;
    // where each bucket begins in the order of buckets, and the place of each diagonal there
    for (int d = threadIdx.x; d < D; d += NT) bucket[d] = mrf_bucket_clamped(P.bucket_of[d], NB);
    __syncthreads();
    for (int b = threadIdx.x; b <= NB; b += NT) {
        int n = 0;
        for (int d = 0; d < D; ++d) n += bucket[d] < b;
        begin[b] = n;
    }
    for (int d = threadIdx.x; d < D; d += NT) {
        int n = 0;
        for (int e = 0; e < D; ++e) n += bucket[e] < bucket[d] || (bucket[e] == bucket[d] && e < d);
        place[d] = n;
    }
    __syncthreads();
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63, groups = P.groups;
    const int mine = lane / K, j = lane - mine * K;
    float *sums = diag[wv];
    T *tile = (T *)(staged + wv * P.tile);
    // the first entry of the tables that the lane sums, the only one for most sizes
    const int item_g = lane / NB, item_b = lane - item_g * NB, item_first = item_g * D + begin[item_b], item_end = item_g * D + begin[item_b + 1];
    quad next[NQ];
    T rest = (T)0.0f;      // the entry behind the last whole chunk that is the lane's
    const auto fetch = [&](long long g0) {
        const int n = (P.G - g0 < groups ? (int)(P.G - g0) : groups) * S, chunks = n / PER;
        const T *from = (const T *)P.dout + (size_t)g0 * S;
#pragma unroll
        for (int i = 0; i < NQ; ++i)
            if (lane + 64 * i < chunks) next[i] = *(const chunk *)(from + (unsigned)(lane + 64 * i) * PER);
        if (chunks * PER + lane < n) rest = from[chunks * PER + lane];
    };
    const long long step = (long long)gridDim.x * MRF_BUCKET_WAVES * groups;
    long long g0 = ((long long)blockIdx.x * MRF_BUCKET_WAVES + wv) * groups;
    if (g0 < P.G) fetch(g0);
    for (; g0 < P.G; g0 += step) {
        const int here = P.G - g0 < groups ? (int)(P.G - g0) : groups, n = here * S, chunks = n / PER;
#pragma unroll
        for (int i = 0; i < NQ; ++i)
            if (lane + 64 * i < chunks) ((quad *)tile)[lane + 64 * i] = next[i];
        if (chunks * PER + lane < n) tile[chunks * PER + lane] = rest;
        if (g0 + step < P.G) fetch(g0 + step);
        mrf_wave_lds_fence();
        if (mine < here) {
            const T *x = tile + mine * S;
            float *to = sums + mine * D;
            int at = j, turn = K - 1 - j, d = j + (Q - 1);      // element; row in which the lane begins again; its diagonal
            float s = 0.0f, done = 0.0f;
            for (int q = 0; q < Q; q += 8) {
                float v[8];
                int t = turn;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[i] = mrf_to_f32(x[q + i < Q ? at : j]);
                    at += q + i == t ? 1 : K + 1;
                    if (!WIDE) t += q + i == t ? K : 0;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (q + i < Q) {
                        s += v[i];
                        if constexpr (WIDE) {
                            done = q + i == turn ? s : done;
                            s = q + i == turn ? 0.0f : s;
                        } else if (q + i == turn) {
                            to[place[d]] = s;
                            s = 0.0f;
                            d -= K;
                            turn += K;
                        }
                    }
            }
            if constexpr (WIDE) {
                // (Q <= K: a lane begins again once at most)
                if (turn < Q) {
                    to[place[d]] = done;
                    d -= K;
                }
                if (turn != Q - 1) to[place[d]] = s;
            } else if (turn - K != Q - 1) {
                to[place[d]] = s;
            }
        }
        mrf_wave_lds_fence();
        for (int i = lane; i < here * NB; i += 64) {
            int g = item_g, b = item_b, d = item_first, last = item_end;
            if (i >= 64) {
                g = i / NB;
                b = i - g * NB;
                d = g * D + begin[b];
                last = g * D + begin[b + 1];
            }
            float s = 0.0f;
#pragma unroll 4
            for (; d < last; ++d) s += sums[d];
            P.dtable[(g0 + g) * P.sg + b * P.sb] = s;
        }
        mrf_wave_lds_fence();
    }
}

// Long matrices: a wavefront goes down a strip of 256 columns, four of them a lane, whole chunks of the matrix, and the sums move instead: after
// four rows, the diagonals that a lane's columns are on are those of the lane before it.  Entry j of row r (of four) is on the lane's
// diagonal j - r: sums 0 .. 3 go to the next lane, and those below 0, the new lane's 1 .. 3, meet them there.  What leaves the last
// lane is complete for the strip.  Eight wavefronts with consecutive rows add up theirs in LDS.  Bound by memory: 16 matrices of 2,048 x 2,048 in 16 bits
// 28 us (4.8 TB/s; a lane per diagonal and loads that move 52), and 4.6 and 3.9 us for the two sums; 1 of 256 x 256 in 32 bits 8.5 us.
constexpr int MRF_BUCKET_STRIP = 256, MRF_BUCKET_STACK = 8, MRF_BUCKET_TQ = 64;      // columns; wavefronts of a workgroup; rows of one at most

// ONE: a workgroup has a whole matrix (256 columns, 512 rows at most), and sums its buckets at once.
template <class T, bool ONE>
__global__ void __launch_bounds__(64 * MRF_BUCKET_STACK) mrf_bucket_bwd_long(const MrfBucketParams P)
{
    typedef typename MrfVec<T, 4>::type vec;
    constexpr int R = 16;      // rows on their way at once
    constexpr int SLOTS = MRF_BUCKET_STRIP + MRF_BUCKET_STACK * MRF_BUCKET_TQ;
    __shared__ float slots[MRF_BUCKET_STACK][MRF_BUCKET_STRIP + MRF_BUCKET_TQ];      // by diagonal, from that of the first column and the last row on
    __shared__ float sums[ONE ? SLOTS : 1];
    __shared__ int bucket[ONE ? SLOTS : 1];
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int Q = P.Q, K = P.K, TQ = P.TQ;
    const int strip = (int)(blockIdx.x % (unsigned)P.strips), part = (int)(blockIdx.x / (unsigned)P.strips);
    const int c0 = strip * MRF_BUCKET_STRIP, c = c0 + 4 * lane, q0 = (part * MRF_BUCKET_STACK + wv) * TQ;
    const int rows = Q - q0 < TQ ? Q - q0 : TQ;
    // (the row's last chunk, where it is not full, is read as the row's last four columns; lanes behind the row read its first)
    const int in = c + 4 <= K ? c : (c < K && K >= 4 ? K - 4 : 0), gone = c < K ? c - in : 4;
    const bool ragged = c0 + MRF_BUCKET_STRIP > K;
    const int n = MRF_BUCKET_STRIP + MRF_BUCKET_STACK * TQ;
    if constexpr (ONE) {
        // slot i is the diagonal i - 8 TQ + Q - 1; those without an entry get no bucket
        for (int i = threadIdx.x; i < n; i += 64 * MRF_BUCKET_STACK) {
            const int d = i - MRF_BUCKET_STACK * TQ + Q - 1;
            bucket[i] = d >= 0 && d < Q + K - 1 ? mrf_bucket_clamped(P.bucket_of[d], P.NB) : -1;
        }
    }
    for (long long g = blockIdx.y; g < P.G; g += gridDim.y) {
        const T *x = (const T *)P.dout + (size_t)g * Q * K;      // (a wavefront may have no row at all: its first is not read then)
        float s[7] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        float *mine = slots[wv];
        for (int q = 0; q < TQ; q += R) {
            vec w[R];
#pragma unroll
            for (int i = 0; i < R; i += 4) {
                if (q + i + 4 <= rows && K >= 4) {
#pragma unroll
                    for (int r = i; r < i + 4; ++r) w[r] = *(const vec *)(x + (long long)(q0 + q + r) * K + (unsigned)in);
                } else if (q + i >= rows) {
#pragma unroll
                    for (int r = i; r < i + 4; ++r)
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[r][j] = (T)0.0f;
                } else {
                    // the last rows, entry by entry (what is not there is read as the matrix's first entry, and not used)
#pragma unroll
                    for (int r = i; r < i + 4; ++r)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const bool there = q + r < rows && (K >= 4 || j < K);
                            w[r][j] = x[there ? (long long)(q0 + q + r) * K + (in + j) : 0];
                        }
                }
            }
            float v[R][4];
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) v[i][j] = q + i < rows ? mrf_to_f32((T)w[i][j]) : 0.0f;
            if (ragged) {
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    v[i][0] = gone == 0 ? v[i][0] : (gone == 1 ? v[i][1] : (gone == 2 ? v[i][2] : (gone == 3 ? v[i][3] : 0.0f)));
                    v[i][1] = gone == 0 ? v[i][1] : (gone == 1 ? v[i][2] : (gone == 2 ? v[i][3] : 0.0f));
                    v[i][2] = gone == 0 ? v[i][2] : (gone == 1 ? v[i][3] : 0.0f);
                    v[i][3] = gone == 0 ? v[i][3] : 0.0f;
                }
                if (K < 4) {
#pragma unroll
                    for (int i = 0; i < R; ++i)
#pragma unroll
                        for (int j = 1; j < 4; ++j) v[i][j] = j < K ? v[i][j] : 0.0f;
                }
            }
#pragma unroll
            for (int i = 0; i < R; i += 4) {
                if (q + i >= TQ) break;
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int j = 0; j < 4; ++j) s[j - r + 3] += v[i + r][j];
                if (lane == 63) {
#pragma unroll
                    for (int t = 0; t < 4; ++t) mine[MRF_BUCKET_STRIP + (TQ - q - i - 4) + t] = s[t + 3];
                }
#pragma unroll
                for (int t = 3; t >= 0; --t) {
                    const float up = __shfl_up(s[t + 3], 1);
                    s[t + 3] = (lane > 0 ? up : 0.0f) + (t > 0 ? s[t - 1] : 0.0f);
                }
                s[0] = s[1] = s[2] = 0.0f;
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) mine[4 * lane + t] = s[t + 3];
        __syncthreads();
        float *out = ONE ? sums : P.diagonals + (((size_t)g * P.T + part) * P.strips + strip) * n;
        for (int i = threadIdx.x; i < n; i += 64 * MRF_BUCKET_STACK) {
            float t = 0.0f;
#pragma unroll
            for (int w = 0; w < MRF_BUCKET_STACK; ++w) {
                const int k = i - (MRF_BUCKET_STACK - 1 - w) * TQ;
                if (k >= 0 && k < MRF_BUCKET_STRIP + TQ) t += slots[w][k];
            }
            out[i] = t;
        }
        __syncthreads();
        if constexpr (ONE) {
            if (P.NB <= 64 * MRF_BUCKET_STACK) {
                // a wavefront per bucket
                for (int b = wv; b < P.NB; b += MRF_BUCKET_STACK) {
                    float t = 0.0f;
                    for (int i = lane; i < n; i += 64) t += bucket[i] == b ? sums[i] : 0.0f;
                    t = mrf_lanes_sum<64>(t);
                    if (lane == 0) P.dtable[g * P.sg + b * P.sb] = t;
                }
            } else {
                // a thread per bucket, most of which are empty
                for (int b = threadIdx.x; b < P.NB; b += 64 * MRF_BUCKET_STACK) {
                    float t = 0.0f;
                    for (int i = 0; i < n; ++i) t += bucket[i] == b ? sums[i] : 0.0f;
                    P.dtable[g * P.sg + b * P.sb] = t;
                }
            }
            __syncthreads();
        }
    }
}

// a thread per diagonal: its sums over the parts and the strips that it crosses (as one kernel with the sum over buckets 10 us instead of 4.6 + 3.9, 16
// matrices of 2,048 x 2,048)
__global__ void __launch_bounds__(256) mrf_bucket_bwd_diagonals(const MrfBucketParams P)
{
    static_assert(MRF_BUCKET_STRIP == 256 && MRF_BUCKET_STACK * MRF_BUCKET_TQ <= 2 * MRF_BUCKET_STRIP, "strips of a diagonal");
    const int Q = P.Q, D = Q + P.K - 1, d = (int)(blockIdx.x * 256 + threadIdx.x), rows = MRF_BUCKET_STACK * P.TQ, n = MRF_BUCKET_STRIP + rows;
    if (d >= D) return;
    // the parts of its rows
    const int off = d - (Q - 1), top = off < 0 ? -off : 0, bottom = Q - 1 < P.K - 1 - off ? Q - 1 : P.K - 1 - off;
    for (long long g = blockIdx.y; g < P.G; g += gridDim.y) {
        const float *x = P.diagonals + (size_t)g * P.T * P.strips * n;
        double s = 0.0;      // (of up to 2^22 parts)
#pragma unroll 4
        for (int p = top / rows; p <= bottom / rows; ++p) {
            // slot i of strip k is the diagonal 256 k + i - (p + 1) rows + Q - 1: in three strips at most
            const int at = d + (p + 1) * rows - (Q - 1), k0 = at >> 8, i0 = at & 255;
#pragma unroll
            for (int v = 0; v < 3; ++v) {
                const int k = k0 - v, i = i0 + v * MRF_BUCKET_STRIP;
                const bool there = k >= 0 && k < P.strips && i < n;
                const float y = x[there ? ((size_t)p * P.strips + k) * n + i : 0];
                s += (double)(there ? y : 0.0f);
            }
        }
        P.totals[g * D + d] = (float)s;
    }
}

// A workgroup per bucket and group: the diagonals of that bucket, four of a thread's looked up at once.  A thread has as many as 2^23 diagonals: its
// sum in 64 bits (in 32, 30 million entries of one sign in one row were off by 2e-4), those of the threads meet in 32.
template <int NT>
__global__ void __launch_bounds__(NT) mrf_bucket_bwd_sum(const MrfBucketParams P)
{
    __shared__ float waves[NT / 64];
    const int D = P.T > 0 ? P.Q + P.K - 1 : 0, b = blockIdx.x;
    for (long long g = blockIdx.y; g < P.G; g += gridDim.y) {
        double own = 0.0;
        for (int first = threadIdx.x; first < D; first += 4 * NT) {
            int bucket[4];
            float total[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int d = first + u * NT;
                bucket[u] = P.bucket_of[d < D ? d : D - 1];
                total[u] = P.totals[g * D + (d < D ? d : D - 1)];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) total[u] = first + u * NT < D && mrf_bucket_clamped(bucket[u], P.NB) == b ? total[u] : 0.0f;
            own += (double)((total[0] + total[1]) + (total[2] + total[3]));
        }
        float s = mrf_lanes_sum<64>((float)own);
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
        __syncthreads();
        if (threadIdx.x < 64) {
            s = mrf_lanes_sum<NT / 64>(threadIdx.x < NT / 64 ? waves[threadIdx.x] : 0.0f);
            if (threadIdx.x == 0) P.dtable[g * P.sg + b * P.sb] = s;
        }
        __syncthreads();
    }
}

using namespace mrf_host;

namespace {

int bucket_check(int64_t G, int32_t Q, int32_t K, int32_t NB)
{
    if (G < 0 || G > 0x7fffffffLL || Q < 0 || K < 0 || NB < 1 || NB > 65536) return MRF_ERR_BAD_SHAPE;
    if ((int64_t)Q + K > LONGEST_ROW || (double)G * Q * K > 1e15) return MRF_ERR_BAD_SHAPE;
    return MRF_OK;
}

// offsets of a map: far from where sums of 64 bits would wrap around
constexpr int64_t FARTHEST = (int64_t)1 << 40;

bool bucket_offsets(int64_t first, int64_t n) { return first >= -FARTHEST && first <= FARTHEST && n >= 0 && n <= FARTHEST; }

// the call's part of the map: every offset k - q - query_offset has to be in it
int bucket_map(int32_t Q, int32_t K, const int32_t *bucket_of, int64_t first_offset, int64_t n_offsets, int64_t query_offset, const int **map)
{
    if (!bucket_offsets(first_offset, n_offsets) || query_offset < -FARTHEST || query_offset > FARTHEST) return MRF_ERR_BAD_ARGUMENT;
    const int64_t lowest = -(int64_t)(Q - 1) - query_offset, highest = (int64_t)(K - 1) - query_offset;
    if (lowest < first_offset || highest > first_offset + n_offsets - 1) return MRF_ERR_BAD_ARGUMENT;
    *map = bucket_of + (lowest - first_offset);
    return MRF_OK;
}

void bucket_strides(MrfBucketParams &P, int heads_last)
{
    P.sg = heads_last ? 1 : P.NB;
    P.sb = heads_last ? P.G : 1;
}

// Small matrices by the wavefront, unless they are few and not very small: then the workgroup's sort of the diagonals is most of the call, and a
// workgroup for each matrix is faster (32-bit square matrices, one against the other: 64 sides 10.5 / 7.5 us for 1 matrix, 11.2 / 9.3 for 512, 15.8 / 29.8
// for 2,048; 32 sides 7.0 / 7.2, 7.7 / 9.3, 7.8 / 27.4; 262,144 of 21 sides 96 / 3,106).
bool bucket_small_backward(const MrfBucketParams &P)
{
    return P.Q <= MRF_BUCKET_SIDE && P.K <= MRF_BUCKET_SIDE && P.NB <= MRF_BUCKET_MANY && (P.G > 512 || (P.Q <= 32 && P.K <= 32));
}

// A workgroup for a whole matrix needs no partial sums: 1,000 of 256 x 256 in 32 bits 56 us, with them 120; 1 such matrix 8.5 and 12.1; 1 of 512 x 256
// 13.2 and 12.9.
bool bucket_one_workgroup(const MrfBucketParams &P) { return P.K <= MRF_BUCKET_STRIP && P.Q <= MRF_BUCKET_STACK * MRF_BUCKET_TQ; }

// Rows of a wavefront (a multiple of four): an eighth of a matrix that a workgroup has as a whole, else 64, or so few that there are 1,024
// wavefronts: four a compute unit read fast enough, and more of them leave more partial sums (32-bit, 64 rows always / 1,024 / 4,096 wavefronts: 1 of
// 2,048 x 2,048 19 / 15 / 25 us, 4 of 600 x 600 25 / 16 / 16, 32 of 300 x 300 25 / 15 / 20).
void bucket_parts(MrfBucketParams &P)
{
    P.strips = (int)(((long long)P.K + MRF_BUCKET_STRIP - 1) / MRF_BUCKET_STRIP);
    P.TQ = MRF_BUCKET_TQ;
    if (bucket_one_workgroup(P)) P.TQ = ((P.Q + MRF_BUCKET_STACK - 1) / MRF_BUCKET_STACK + 3) / 4 * 4;
    else
        while (P.TQ > 4 && P.G * P.strips * ((P.Q + P.TQ - 1LL) / P.TQ) < 1024) P.TQ /= 2;
    P.T = (int)((P.Q + (long long)MRF_BUCKET_STACK * P.TQ - 1) / (MRF_BUCKET_STACK * P.TQ));
}

// Many small matrices by whole chunks.  Few of them (below 4,096, or in 32 bits up to 16,384, in 16 bits up to 8,192, of nearly 64 x 64 whose rows are whole
// chunks) are faster row by row from a line, where no thread has an index to work out first.  Calls one behind the other, chunks / lines, 32 bits: 2,048 of 16 x 16 4.0 /
// 3.9 us, of 64 x 64 21 / 9.5; 16,384 of 56 x 56 42 / 39, of 64 x 64 57 / 49, of 63 x 63 58 / 68, of 24 x 24 12 / 26; 262,144 of 21 x 21 92 to 103 / 309.
// 16 bits: 2,048 of 64 x 64 19 / 7.1; 4,096 of 56 x 56 17.6 / 13.8; 8,192 of 56 x 56 21.4 / 21.5, of 64 x 64 25 / 21.5; 16,384 of 56 x 56 27 / 35, of 64 x 64
// 32 / 35; 262,144 of 21 x 21 50 / 366.
bool bucket_small_forward(const MrfBucketParams &P, int V)
{
    const long long S = (long long)P.Q * P.K;
    if (S > MRF_BUCKET_SMALL || P.NB > MRF_BUCKET_LDS / 4 || P.G < 4096) return false;
    return !(S >= 56 * 56 && P.K % V == 0 && P.G <= (V == 4 ? 16384 : 8192));
}

template <class T> int bucket_forward(MrfBucketParams P, hipStream_t st)
{
    const long long S = (long long)P.Q * P.K;
    const unsigned groups = (unsigned)(P.G < 65535 ? P.G : 65535);
    constexpr int V = 16 / (int)sizeof(T);
    if (bucket_small_forward(P, V)) {
        // 16 fours of matrices a workgroup, or so many that the tables have room, and that the launch has many a workgroup (of 1,024 threads: 25,000 of 63 x 63
        // 88 us instead of 100) or fills the machine (of 256)
        P.quads = 16;
        while (P.quads > 1 && (P.quads * 4 * P.NB > MRF_BUCKET_LDS || P.G < (S <= 256 * MRF_BUCKET_CHUNKS ? 2048LL : 16384LL) * P.quads)) P.quads /= 2;
        const long long need = (P.G + 4 * P.quads - 1) / (4 * P.quads);
        // (256 threads where their chunks suffice: 2.4 million of 5 x 5 120 us, 355 with 1,024, of which 25 have work; 262,144 of 21 x 21,
        // calls one behind the other, 103 to 107 and 101)
        if (S <= 256 * MRF_BUCKET_CHUNKS)
            hipLaunchKernelGGL((mrf_bucket_fwd_small<T, 256>), dim3((unsigned)(need < 2048 ? need : 2048)), dim3(256), 0, st, P);
        else
            hipLaunchKernelGGL((mrf_bucket_fwd_small<T, 1024>), dim3((unsigned)(need < 512 ? need : 512)), dim3(1024), 0, st, P);
        return launch_status("mrf_bucket_fwd_small");
    }
    P.KL = 1;
    while (P.KL < 64 && P.KL * V < P.K) P.KL *= 2;
    const int runs = 64 / P.KL;
    P.TR = MRF_BUCKET_RUNS / runs < 32 ? MRF_BUCKET_RUNS / runs : 32;
    long long tiles;
    for (;; P.TR /= 2) {
        const long long W = (long long)P.KL * V, TQ = (long long)P.TR * runs;
        tiles = ((P.K + W - 1) / W) * ((P.Q + TQ - 1) / TQ);
        if (P.TR <= 1 || P.G * tiles >= 4096) break;
    }
    if (tiles > 0x7fffffffLL) return MRF_ERR_BAD_SHAPE;
    hipLaunchKernelGGL((mrf_bucket_fwd_long<T, V>), dim3((unsigned)((tiles + 3) / 4), groups), dim3(256), 0, st, P);
    return launch_status("mrf_bucket_fwd_long");
}

// 1,024 threads for a bucket, 256 where there are more than 1,024 buckets in all and starting so many large workgroups takes longest (backward calls, 64
// groups of 300 x 300 and 64 buckets 25.7 / 19.8 us, 23 of 29 x 4,702 18.3 / 16.8; 4 of 300 x 600 and 16 buckets 14.0 / 15.2).
int bucket_sum(const MrfBucketParams &P, hipStream_t st)
{
    const dim3 grid((unsigned)P.NB, (unsigned)(P.G < 65535 ? P.G : 65535));
    if (P.G * P.NB > 1024) hipLaunchKernelGGL(mrf_bucket_bwd_sum<256>, grid, dim3(256), 0, st, P);
    else hipLaunchKernelGGL(mrf_bucket_bwd_sum<1024>, grid, dim3(1024), 0, st, P);
    return launch_status("mrf_bucket_bwd_sum");
}

template <class T> int bucket_backward(MrfBucketParams P, hipStream_t st)
{
    if (bucket_small_backward(P)) {
        const int fit = 64 / P.K, room = MRF_BUCKET_DIAG / (P.Q + P.K - 1);
        P.groups = fit < room ? fit : room;
        P.tile = (P.groups * P.Q * P.K * (int)sizeof(T) + 15) / 16 * 16;
        // (no more workgroups than run at once: each sorts the diagonals first)
        const long long need = (P.G + MRF_BUCKET_WAVES * P.groups - 1) / (MRF_BUCKET_WAVES * P.groups);
        const int lds = MRF_BUCKET_WAVES * (P.tile + 4 * MRF_BUCKET_DIAG) + 16 * MRF_BUCKET_SIDE + 4 * MRF_BUCKET_MANY + 16;
        const int most = 256 * (160 * 1024 / lds < 16 ? 160 * 1024 / lds : 16);
        const dim3 grid((unsigned)(need < most ? need : most)), block(64 * MRF_BUCKET_WAVES);
        const unsigned shared = (unsigned)(MRF_BUCKET_WAVES * P.tile);
        if (P.tile <= 8 * 64 * 16) {
            if (P.Q <= P.K) hipLaunchKernelGGL((mrf_bucket_bwd_small<T, true, 8>), grid, block, shared, st, P);
            else hipLaunchKernelGGL((mrf_bucket_bwd_small<T, false, 8>), grid, block, shared, st, P);
        } else {
            if (P.Q <= P.K) hipLaunchKernelGGL((mrf_bucket_bwd_small<T, true, 16>), grid, block, shared, st, P);
            else hipLaunchKernelGGL((mrf_bucket_bwd_small<T, false, 16>), grid, block, shared, st, P);
        }
        return launch_status("mrf_bucket_bwd_small");
    }
    bucket_parts(P);
    const unsigned groups = (unsigned)(P.G < 65535 ? P.G : 65535);
    if (bucket_one_workgroup(P)) {
        hipLaunchKernelGGL((mrf_bucket_bwd_long<T, true>), dim3(1, groups), dim3(64 * MRF_BUCKET_STACK), 0, st, P);
        return launch_status("mrf_bucket_bwd_long");
    }
    P.totals = P.diagonals + (size_t)P.G * P.T * P.strips * (MRF_BUCKET_STRIP + MRF_BUCKET_STACK * (size_t)P.TQ);
    const long long blocks = (long long)P.strips * P.T;
    if (blocks > 0x7fffffffLL) return MRF_ERR_BAD_SHAPE;
    hipLaunchKernelGGL((mrf_bucket_bwd_long<T, false>), dim3((unsigned)blocks, groups), dim3(64 * MRF_BUCKET_STACK), 0, st, P);
    int rc = launch_status("mrf_bucket_bwd_long");
    if (rc != MRF_OK) return rc;
    hipLaunchKernelGGL(mrf_bucket_bwd_diagonals, dim3((unsigned)(((long long)P.Q + P.K - 1 + 255) / 256), groups), dim3(256), 0, st, P);
    rc = launch_status("mrf_bucket_bwd_diagonals");
    return rc != MRF_OK ? rc : bucket_sum(P, st);
}

}  // namespace

extern "C" {

int mrf_distance_buckets(int32_t n_buckets, int64_t far_distance, int two_sided, int64_t first_offset, int64_t n_offsets, int32_t *bucket_of)
{
    if (n_buckets < 1 || n_buckets > 65536 || far_distance < 1 || !bucket_offsets(first_offset, n_offsets)) return MRF_ERR_BAD_ARGUMENT;
    if (n_offsets == 0) return MRF_OK;
    if (!bucket_of) return MRF_ERR_NULL_POINTER;
    const int side = two_sided && n_buckets > 1 ? n_buckets / 2 : n_buckets;      // buckets of one sign
    const int single = side / 2 > 1 ? side / 2 : 1;                               // distances with a bucket of their own
    const double far = far_distance > single ? (double)far_distance : (double)(single + 1);
    const double scale = (side - single) / log(far / single);
    for (int64_t i = 0; i < n_offsets; ++i) {
        const int64_t d = first_offset + i;
        const int64_t n = d < 0 ? -d : (two_sided ? d : 0);
        // (a distance that lies on a boundary belongs to the upper bucket: the small term is far above the logarithm's rounding and far
        // below what one label more makes)
        int64_t b = n < single ? n : single + (int64_t)floor(log((double)n / single) * scale + 1e-9);
        if (b > side - 1) b = side - 1;
        bucket_of[i] = (int32_t)(b + (two_sided && n_buckets > 1 && d > 0 ? n_buckets - side : 0));
    }
    return MRF_OK;
}

size_t mrf_bucket_pairwise_workspace_bytes(int64_t n_groups, int32_t Q, int32_t K, int32_t n_buckets)
{
    if (bucket_check(n_groups, Q, K, n_buckets) != MRF_OK) return 0;
    MrfBucketParams P = {};
    P.G = n_groups; P.Q = Q; P.K = K; P.NB = n_buckets;
    if (n_groups == 0 || Q == 0 || K == 0 || bucket_small_backward(P) || bucket_one_workgroup(P)) return 256;
    bucket_parts(P);
    return sizeof(float) * (size_t)n_groups *
           ((size_t)P.T * (size_t)P.strips * (MRF_BUCKET_STRIP + MRF_BUCKET_STACK * (size_t)P.TQ) + (size_t)Q + K - 1);
}

int mrf_bucket_pairwise_forward(int64_t n_groups, int32_t Q, int32_t K, int32_t n_buckets, const float *table, int heads_last,
                                const int32_t *bucket_of, int64_t first_offset, int64_t n_offsets, int64_t query_offset, void *out,
                                int out_type, void *hip_stream)
{
    int rc = bucket_check(n_groups, Q, K, n_buckets);
    if (rc != MRF_OK) return rc;
    if (!known_type(out_type)) return MRF_ERR_BAD_ARGUMENT;
    if (n_groups == 0 || Q == 0 || K == 0) return MRF_OK;
    if (!table || !bucket_of || !out) return MRF_ERR_NULL_POINTER;
    MrfBucketParams P = {};
    rc = bucket_map(Q, K, bucket_of, first_offset, n_offsets, query_offset, &P.bucket_of);
    if (rc != MRF_OK) return rc;
    P.G = n_groups; P.Q = Q; P.K = K; P.NB = n_buckets; P.table = table; P.out = out;
    bucket_strides(P, heads_last);
    hipStream_t st = (hipStream_t)hip_stream;
    if (out_type == MRF_F32) return bucket_forward<float>(P, st);
    return out_type == MRF_F16 ? bucket_forward<mrf_f16>(P, st) : bucket_forward<mrf_bf16>(P, st);
}

int mrf_bucket_pairwise_backward(int64_t n_groups, int32_t Q, int32_t K, int32_t n_buckets, const void *grad_out, int out_type,
                                 int heads_last, const int32_t *bucket_of, int64_t first_offset, int64_t n_offsets, int64_t query_offset,
                                 float *grad_table, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    int rc = bucket_check(n_groups, Q, K, n_buckets);
    if (rc != MRF_OK) return rc;
    if (!known_type(out_type)) return MRF_ERR_BAD_ARGUMENT;
    if (n_groups == 0) return MRF_OK;
    if (!grad_table) return MRF_ERR_NULL_POINTER;
    MrfBucketParams P = {};
    P.G = n_groups; P.Q = Q; P.K = K; P.NB = n_buckets; P.dout = grad_out; P.dtable = grad_table;
    bucket_strides(P, heads_last);
    hipStream_t st = (hipStream_t)hip_stream;
    if (Q == 0 || K == 0) return bucket_sum(P, st);      // no entry of the matrix: sums over no part
    if (!grad_out || !bucket_of || !workspace) return MRF_ERR_NULL_POINTER;
    if (workspace_bytes < mrf_bucket_pairwise_workspace_bytes(n_groups, Q, K, n_buckets)) return MRF_ERR_WORKSPACE_TOO_SMALL;
    rc = bucket_map(Q, K, bucket_of, first_offset, n_offsets, query_offset, &P.bucket_of);
    if (rc != MRF_OK) return rc;
    P.diagonals = (float *)workspace;
    if (out_type == MRF_F32) return bucket_backward<float>(P, st);
    return out_type == MRF_F16 ? bucket_backward<mrf_f16>(P, st) : bucket_backward<mrf_bf16>(P, st);
}

}  // extern "C"
