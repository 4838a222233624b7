// Pairwise functions from a table of label distances in buckets, and the table's gradient (see
// mrf_bucket_pairwise_forward in the header for the formulas).
#include "mrfmp_rows.h"

struct MrfBucketParams {
    long long G;
    int Q, K, NB;
    const float *table;
    long long sg, sb;            // strides of the table: group, bucket
    const int *bucket_of;        // [Q + K - 1] buckets of the offsets from -(Q - 1) - query_offset on
    void *out;                   // forward [G][Q][K]
    const void *dout;            // backward
    float *dtable;
    float *diagonals;            // [G][T][Q + K - 1] sums over the rows of a part (long matrices)
    int quads;                   // forward, many small matrices: fours of groups whose tables are in LDS at once
    int KL, TR;                  // forward, long matrices: lanes of a row, rows of a lane
    int T, TQ;                   // backward, long matrices: parts of TQ rows
};

__device__ inline int mrf_bucket_clamped(int b, int NB) { return b < 0 ? 0 : (b < NB ? b : NB - 1); }

// ---- forward, many small matrices (Q K <= 4096).  Four matrices are Q K chunks of four entries, whatever Q and K: a thread keeps the places in
// the tables of the four entries of its chunks, in registers, and goes from four matrices to the next.  Chunks of neighbouring threads
// are neighbours in memory, and no index is computed twice.
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
// in LDS, and a lane that goes down V columns reads one new value a row.  KL lanes share a row, 64 / KL runs of TR rows a wavefront.
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

// Many small matrices (Q, K <= 64): lanes j < K of a matrix go down its rows from column j on and begin again at column 0, so that none idles: a
// wavefront takes as many matrices as have room.  Where a lane begins again, a diagonal's sum is complete.
constexpr int MRF_BUCKET_SIDE = 64, MRF_BUCKET_DIAG = 1024, MRF_BUCKET_MANY = 1024;      // Q, K; diagonals of a wavefront; buckets

template <class T>
__global__ void __launch_bounds__(256) mrf_bucket_bwd_small(const MrfBucketParams P)
{
    __shared__ float diag[4][MRF_BUCKET_DIAG];
    __shared__ int bucket[2 * MRF_BUCKET_SIDE], order[2 * MRF_BUCKET_SIDE], begin[MRF_BUCKET_MANY + 1];
    const int Q = P.Q, K = P.K, NB = P.NB, S = Q * K, D = Q + K - 1;
    // the diagonals in the order of their buckets, and where each bucket begins
    for (int d = threadIdx.x; d < D; d += 256) bucket[d] = mrf_bucket_clamped(P.bucket_of[d], NB);
    __syncthreads();
    for (int b = threadIdx.x; b <= NB; b += 256) {
        int n = 0;
        for (int d = 0; d < D; ++d) n += bucket[d] < b;
        begin[b] = n;
    }
    for (int d = threadIdx.x; d < D; d += 256) {
        int n = 0;
        for (int e = 0; e < D; ++e) n += bucket[e] < bucket[d] || (bucket[e] == bucket[d] && e < d);
        order[n] = d;
    }
    __syncthreads();
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int fit = 64 / K, room = MRF_BUCKET_DIAG / D, groups = fit < room ? fit : room;
    const int mine = lane / K, j = lane - mine * K;
    float *sums = diag[wv];
    for (long long g0 = ((long long)blockIdx.x * 4 + wv) * groups; g0 < P.G; g0 += (long long)gridDim.x * 4 * groups) {
        const int here = P.G - g0 < groups ? (int)(P.G - g0) : groups;
        if (mine < here) {
            const T *x = (const T *)P.dout + (size_t)(g0 + mine) * S;
            int k = j, write = mine * D + j + (Q - 1);      // place of the diagonal that the lane is on
            float s = 0.0f;
            for (int q = 0; q < Q; q += 8) {
                T v[8];
                int c = k;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (q + i < Q) v[i] = x[(q + i) * K + c];
                    c = c + 1 == K ? 0 : c + 1;
                }
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (q + i < Q) {
                        s += mrf_to_f32(v[i]);
                        if (++k == K) {
                            sums[write] = s;
                            s = 0.0f;
                            k = 0;
                            write -= K;
                        }
                    }
            }
            if (k > 0) sums[write] = s;
        }
        mrf_wave_lds_fence();
        for (int i = lane; i < here * NB; i += 64) {
            const int g = i / NB, b = i - g * NB;
            float s = 0.0f;
            for (int d = begin[b]; d < begin[b + 1]; ++d) s += sums[g * D + order[d]];
            P.dtable[(g0 + g) * P.sg + b * P.sb] = s;
        }
        mrf_wave_lds_fence();
    }
}

// Long matrices: a wavefront takes 64 neighbouring diagonals through the rows of a part; a lane's rows are those in which its diagonal has a
// column.
template <class T>
__global__ void __launch_bounds__(256) mrf_bucket_bwd_long(const MrfBucketParams P)
{
    const int wv = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int Q = P.Q, K = P.K, D = Q + K - 1;
    const unsigned tiles = (unsigned)((D + 255) / 256);
    const int part = (int)(blockIdx.x / tiles), d0 = (int)(blockIdx.x % tiles) * 256 + wv * 64;
    if (d0 >= D) return;
    const int d = d0 + lane, off = d - (Q - 1);      // column = row + off
    const int q0 = part * P.TQ, q1 = Q - q0 < P.TQ ? Q : q0 + P.TQ;
    // the wavefront's rows; those in which every lane has a column
    const int offlast = (d0 + 63 < D ? d0 + 63 : D - 1) - (Q - 1), off0 = d0 - (Q - 1);
    const int from = q0 > -offlast ? q0 : -offlast, to = q1 < K - off0 ? q1 : K - off0;
    const bool whole = d0 + 63 < D;
    const int in0 = whole ? (from > -off0 ? from : -off0) : to, in1 = whole ? (to < K - offlast ? to : K - offlast) : to;
    for (long long g = blockIdx.y; g < P.G; g += gridDim.y) {
        const T *x = (const T *)P.dout + (size_t)g * Q * K;
        float s = 0.0f;
        const auto some = [&](int a, int b) {
            for (int q = a; q < b; ++q) {
                const int k = q + off;
                if (d < D && k >= 0 && k < K) s += mrf_to_f32(x[(size_t)q * K + k]);
            }
        };
        if (in0 < in1) {
            some(from, in0);
            int q = in0;
            for (; q + 16 <= in1; q += 16) {
                T v[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = x[(size_t)(q + i) * K + (q + i + off)];
                float a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int i = 0; i < 16; ++i) a[i & 3] += mrf_to_f32(v[i]);
                s += (a[0] + a[1]) + (a[2] + a[3]);
            }
            some(q, to);
        } else {
            some(from, to);
        }
        if (d < D) P.diagonals[((size_t)g * P.T + part) * D + d] = s;
    }
}

// a workgroup per bucket and group: the diagonals of that bucket, over the parts in order
__global__ void __launch_bounds__(256) mrf_bucket_bwd_sum(const MrfBucketParams P)
{
    __shared__ float waves[4];
    const int D = P.Q + P.K - 1, b = blockIdx.x;
    for (long long g = blockIdx.y; g < P.G; g += gridDim.y) {
        const float *x = P.diagonals + (size_t)g * P.T * D;
        float s = 0.0f;
        if (P.T > 0)
            for (int d = threadIdx.x; d < D; d += 256)
                if (mrf_bucket_clamped(P.bucket_of[d], P.NB) == b)
                    for (int t = 0; t < P.T; ++t) s += x[(size_t)t * D + d];
        s = mrf_lanes_sum<64>(s);
        if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
        __syncthreads();
        if (threadIdx.x == 0) P.dtable[g * P.sg + b * P.sb] = (waves[0] + waves[1]) + (waves[2] + waves[3]);
        __syncthreads();
    }
}

using namespace mrf_host;

namespace {

int bucket_check(int64_t G, int32_t Q, int32_t K, int32_t NB)
{
    if (G < 0 || G > 0x7fffffffLL || Q < 0 || K < 0 || NB < 1 || NB > 65536) return MRF_ERR_BAD_SHAPE;
    if ((int64_t)Q + K > 0x7fffffffLL || (double)G * Q * K > 1e15) return MRF_ERR_BAD_SHAPE;
    return MRF_OK;
}

// the call's part of the map: every offset k - q - query_offset has to be in it
int bucket_map(int32_t Q, int32_t K, const int32_t *bucket_of, int64_t first_offset, int64_t n_offsets, int64_t query_offset, const int **map)
{
    const int64_t far = (int64_t)1 << 40;
    if (first_offset < -far || first_offset > far || n_offsets < 0 || n_offsets > far || query_offset < -far || query_offset > far)
        return MRF_ERR_BAD_ARGUMENT;
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

bool bucket_small_backward(const MrfBucketParams &P) { return P.Q <= MRF_BUCKET_SIDE && P.K <= MRF_BUCKET_SIDE && P.NB <= MRF_BUCKET_MANY; }

// parts of the rows: about 8,192 wavefronts in all, of at least 32 rows
void bucket_parts(MrfBucketParams &P)
{
    const long long D = (long long)P.Q + P.K - 1, columns = P.G * ((D + 63) / 64), most = (P.Q + 31) / 32;
    long long t = (8192 + columns - 1) / columns;
    t = t < most ? t : most;
    P.TQ = (int)((P.Q + t - 1) / t);
    P.T = (P.Q + P.TQ - 1) / P.TQ;
}

template <class T> int bucket_forward(MrfBucketParams P, hipStream_t st)
{
    const long long S = (long long)P.Q * P.K;
    const unsigned groups = (unsigned)(P.G < 65535 ? P.G : 65535);
    if (S <= MRF_BUCKET_SMALL && P.NB <= MRF_BUCKET_LDS / 4) {
        P.quads = 16;
        while (P.quads > 1 && (P.quads * 4 * P.NB > MRF_BUCKET_LDS || (P.G + 2 * P.quads - 1) / (2 * P.quads) < 1024)) P.quads /= 2;
        const long long need = (P.G + 4 * P.quads - 1) / (4 * P.quads);
        if (S <= 256 * MRF_BUCKET_CHUNKS)
            hipLaunchKernelGGL((mrf_bucket_fwd_small<T, 256>), dim3((unsigned)(need < 2048 ? need : 2048)), dim3(256), 0, st, P);
        else
            hipLaunchKernelGGL((mrf_bucket_fwd_small<T, 1024>), dim3((unsigned)(need < 512 ? need : 512)), dim3(1024), 0, st, P);
        return launch_status("mrf_bucket_fwd_small");
    }
    constexpr int V = 16 / (int)sizeof(T);
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

int bucket_sum(const MrfBucketParams &P, hipStream_t st)
{
    hipLaunchKernelGGL(mrf_bucket_bwd_sum, dim3((unsigned)P.NB, (unsigned)(P.G < 65535 ? P.G : 65535)), dim3(256), 0, st, P);
    return launch_status("mrf_bucket_bwd_sum");
}

template <class T> int bucket_backward(MrfBucketParams P, hipStream_t st)
{
    if (bucket_small_backward(P)) {
        const int fit = 64 / P.K, room = MRF_BUCKET_DIAG / (P.Q + P.K - 1), groups = 4 * (fit < room ? fit : room);
        const long long need = (P.G + groups - 1) / groups;
        hipLaunchKernelGGL(mrf_bucket_bwd_small<T>, dim3((unsigned)(need < 2048 ? need : 2048)), dim3(256), 0, st, P);
        return launch_status("mrf_bucket_bwd_small");
    }
    bucket_parts(P);
    const long long tiles = ((long long)P.Q + P.K - 1 + 255) / 256 * P.T;
    hipLaunchKernelGGL(mrf_bucket_bwd_long<T>, dim3((unsigned)tiles, (unsigned)(P.G < 65535 ? P.G : 65535)), dim3(256), 0, st, P);
    const int rc = launch_status("mrf_bucket_bwd_long");
    return rc != MRF_OK ? rc : bucket_sum(P, st);
}

}  // namespace

extern "C" {

int mrf_distance_buckets(int32_t n_buckets, int64_t far_distance, int two_sided, int64_t first_offset, int64_t n_offsets, int32_t *bucket_of)
{
    if (n_buckets < 1 || n_buckets > 65536 || far_distance < 1 || n_offsets < 0) return MRF_ERR_BAD_ARGUMENT;
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
    if (n_groups == 0 || Q == 0 || K == 0 || bucket_small_backward(P)) return 256;
    bucket_parts(P);
    return sizeof(float) * (size_t)n_groups * (size_t)P.T * ((size_t)Q + K - 1);
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
