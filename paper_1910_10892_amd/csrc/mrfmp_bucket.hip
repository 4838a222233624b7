// Pairwise functions from a table of label distances in buckets, and the table's gradient (see
// mrf_bucket_pairwise_forward in the header for the formulas).
#include "mrfmp_learn.h"

struct MrfBucketParams {
    long long G;
    int Q, K, NB;
    const float *table;
    long long sg, sb;            // strides of the table: group, bucket
    const int *bucket_of;        // [..] bucket of the offset -(Q - 1) - query_offset first
    void *out;                   // forward [G][Q][K]
    const void *dout;            // backward
    float *dtable;
    float *partial;              // [G][tiles][NB], or NULL with one tile per group
    int TQ, TK, tiles_q, tiles_k;
};

__device__ inline int mrf_bucket_clamped(int b, int NB) { return b < 0 ? 0 : (b < NB ? b : NB - 1); }

// ---- a thread per element
template <class T>
__global__ void __launch_bounds__(256) mrf_bucket_fwd_any(const MrfBucketParams P)
{
    const long long S = (long long)P.Q * P.K, total = P.G * S;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < total; e += (long long)gridDim.x * 256) {
        const long long g = e / S, r = e - g * S;
        const int q = (int)(r / P.K), k = (int)(r - (long long)q * P.K);
        const int b = mrf_bucket_clamped(P.bucket_of[(long long)k - q + (P.Q - 1)], P.NB);
        ((T *)P.out)[e] = mrf_from_f32<T>(P.table[g * P.sg + b * P.sb]);
    }
}

// ---- backward: a workgroup per tile of TQ rows and TK columns of a group.  A thread walks down a diagonal: in row q it
// takes column (q + j) mod (columns), so that the threads of a wavefront read neighbours and a diagonal's sum stays in a register;
// where the column wraps, the sum of one diagonal is complete and that of the next begins.
constexpr int MRF_BUCKET_TQ = 64, MRF_BUCKET_TK = 256;

template <class T>
__global__ void __launch_bounds__(256) mrf_bucket_bwd_any(const MrfBucketParams P)
{
    __shared__ float diag[MRF_BUCKET_TQ + MRF_BUCKET_TK];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const long long tiles = (long long)P.tiles_q * P.tiles_k;
    for (long long t = blockIdx.x; t < P.G * tiles; t += gridDim.x) {
        const long long g = t / tiles;
        const int ti = (int)(t - g * tiles), tr = ti / P.tiles_k;
        const int q0 = tr * P.TQ, k0 = (ti - tr * P.tiles_k) * P.TK;
        const int tq = P.Q - q0 < P.TQ ? P.Q - q0 : P.TQ, tk = P.K - k0 < P.TK ? P.K - k0 : P.TK;
        const T *x = (const T *)P.dout + ((size_t)g * P.Q + q0) * P.K + k0;
        for (int j = threadIdx.x; j < tk; j += 256) {
            float s = 0.0f;
            int k = j;
            for (int q = 0; q < tq; ++q) {
                s += mrf_to_f32(x[(size_t)q * P.K + k]);
                if (++k == tk) {
                    diag[k - 1 - q + tq - 1] = s;
                    s = 0.0f;
                    k = 0;
                }
            }
            if (k > 0) diag[k - 1] = s;      // offset (k - 1) - (tq - 1)
        }
        __syncthreads();
        const int *bucket_of = P.bucket_of + ((long long)k0 - q0 - (tq - 1) + (P.Q - 1));
        const int n = tq + tk - 1;
        for (int b = wv; b < P.NB; b += 4) {
            float s = 0.0f;
            for (int d = lane; d < n; d += 64)
                if (mrf_bucket_clamped(bucket_of[d], P.NB) == b) s += diag[d];
            s = mrf_lanes_sum<64>(s);
            if (lane == 0) {
                if (P.partial) P.partial[t * P.NB + b] = s;
                else P.dtable[g * P.sg + b * P.sb] = s;
            }
        }
        __syncthreads();
    }
}

// a thread per entry of the table: the tiles of its group in order
__global__ void __launch_bounds__(256) mrf_bucket_sum_any(const MrfBucketParams P)
{
    const long long tiles = (long long)P.tiles_q * P.tiles_k, total = P.G * P.NB;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < total; e += (long long)gridDim.x * 256) {
        const long long g = e / P.NB, b = e - g * P.NB;
        float s = 0.0f;
        for (long long t = 0; t < tiles; ++t) s += P.partial[(g * tiles + t) * P.NB + b];
        P.dtable[g * P.sg + b * P.sb] = s;
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

void bucket_tiles(MrfBucketParams &P)
{
    P.TQ = MRF_BUCKET_TQ;
    P.TK = MRF_BUCKET_TK;
    P.tiles_q = (P.Q + P.TQ - 1) / P.TQ;
    P.tiles_k = (P.K + P.TK - 1) / P.TK;
}

template <class T> int bucket_forward(const MrfBucketParams &P, hipStream_t st)
{
    const long long blocks = (P.G * P.Q * P.K + 255) / 256;
    hipLaunchKernelGGL(mrf_bucket_fwd_any<T>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, st, P);
    return launch_status("mrf_bucket_fwd");
}

template <class T> int bucket_backward(const MrfBucketParams &P, hipStream_t st)
{
    const long long tiles = (long long)P.tiles_q * P.tiles_k, blocks = P.G * tiles;
    hipLaunchKernelGGL(mrf_bucket_bwd_any<T>, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, st, P);
    const int rc = launch_status("mrf_bucket_bwd");
    if (rc != MRF_OK || !P.partial) return rc;
    const long long sums = (P.G * P.NB + 255) / 256;
    hipLaunchKernelGGL(mrf_bucket_sum_any, dim3((unsigned)(sums < 65536 ? sums : 65536)), dim3(256), 0, st, P);
    return launch_status("mrf_bucket_sum");
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
    bucket_tiles(P);
    const size_t tiles = (size_t)P.tiles_q * P.tiles_k;
    return tiles > 1 ? sizeof(float) * (size_t)n_groups * tiles * (size_t)n_buckets : 256;
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
    if (Q == 0 || K == 0) {
        // no entry of the matrix: the sum over no tiles
        hipLaunchKernelGGL(mrf_bucket_sum_any, dim3((unsigned)((P.G * P.NB + 255) / 256 < 65536 ? (P.G * P.NB + 255) / 256 : 65536)), dim3(256), 0, st, P);
        return launch_status("mrf_bucket_sum");
    }
    if (!grad_out || !bucket_of || !workspace) return MRF_ERR_NULL_POINTER;
    if (workspace_bytes < mrf_bucket_pairwise_workspace_bytes(n_groups, Q, K, n_buckets)) return MRF_ERR_WORKSPACE_TOO_SMALL;
    rc = bucket_map(Q, K, bucket_of, first_offset, n_offsets, query_offset, &P.bucket_of);
    if (rc != MRF_OK) return rc;
    bucket_tiles(P);
    if ((long long)P.tiles_q * P.tiles_k > 1) P.partial = (float *)workspace;
    if (out_type == MRF_F32) return bucket_backward<float>(P, st);
    return out_type == MRF_F16 ? bucket_backward<mrf_f16>(P, st) : bucket_backward<mrf_bf16>(P, st);
}

}  // extern "C"
