// Log-probabilities of labels under the SoftMin of the final costs, and the clipped policy loss with its gradient with
// respect to the costs (see mrf_softmin_policy in the header for the formulas).
#include "mrfmp_learn.h"

constexpr int MRF_POLICY_BLOCKS = 4096;      // workgroups at most: partial sums of the loss
constexpr int MRF_POLICY_COUNTS = 256;       // workgroups that count the mask

struct MrfPolicyParams {
    long long N;
    int L;
    const void *cost;
    const void *labels;          // [N] of label_bytes bytes
    int label_bytes;
    const float *advantage;      // entry i / per
    long long per;
    const float *old_logp, *ref_logp;
    const uint8_t *mask;
    float low, high;             // bounds of the ratio
    float kl, scale;             // weight of the KL term, factor on the gradient
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

// the same for probabilities, which may be that small: 2^(t + 64) 2^-64 there
__device__ inline float mrf_exp_small(float x)
{
    const float t = x * 1.44269504088896340736f;
    const bool small = t < -126.0f;
    return __builtin_amdgcn_exp2f(small ? t + 64.0f : t) * (small ? 0x1p-64f : 1.0f);
}

// what a pixel adds to the two sums, and the slope of the loss in its log-probability (before 1 / n)
__device__ inline void mrf_policy_terms(const MrfPolicyParams &P, long long i, float lp, float &gain, float &div, float &slope)
{
    const float A = P.advantage[P.per == 1 ? i : i / P.per];
    const float r = P.old_logp ? expf(lp - P.old_logp[i]) : 1.0f;
    const float open = r * A, held = fminf(fmaxf(r, P.low), P.high) * A;
    gain = fminf(open, held);
    slope = open <= held ? -open : 0.0f;
    div = 0.0f;
    if (P.ref_logp) {
        const float d = P.ref_logp[i] - lp, em = expm1f(d);
        div = em - d;
        if (P.kl > 0.0f) slope -= P.kl * em;
    }
}

__global__ void __launch_bounds__(1024) mrf_policy_count(const MrfPolicyParams P)
{
    __shared__ int waves[16];
    int c = 0;
    for (long long i = (long long)blockIdx.x * 1024 + threadIdx.x; i < P.N; i += (long long)gridDim.x * 1024) c += P.mask[i] != 0;
    for (int m = 1; m < 64; m <<= 1) c += __shfl_xor(c, m);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = c;
    __syncthreads();
    if (threadIdx.x == 0) {
        long long t = 0;
        for (int w = 0; w < 16; ++w) t += waves[w];
        P.counts[blockIdx.x] = t;
    }
}

// number of counted pixels, at least 1; every thread of a workgroup of 256 calls it
__device__ inline long long mrf_policy_counted(const MrfPolicyParams &P, int blocks)
{
    __shared__ long long total;
    if (!P.mask) return P.N > 0 ? P.N : 1;
    if (threadIdx.x < 64) {
        long long c = 0;
        for (int k = threadIdx.x; k < blocks; k += 64) c += P.counts[k];
        for (int m = 1; m < 64; m <<= 1) c += __shfl_xor(c, m);
        if (threadIdx.x == 0) total = c > 0 ? c : 1;
    }
    __syncthreads();
    return total;
}

// ---- a wavefront per row: any length, any alignment.  The first pass keeps a running minimum and the sum under it
template <class T, bool TRAIN>
__global__ void __launch_bounds__(256) mrf_policy_any(const MrfPolicyParams P, int count_blocks)
{
    __shared__ double sums[2][4];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const float inv_n = TRAIN ? 1.0f / (float)mrf_policy_counted(P, count_blocks) : 0.0f;
    double total_gain = 0.0, total_div = 0.0;
    for (long long i = (long long)blockIdx.x * 4 + wv; i < P.N; i += (long long)gridDim.x * 4) {
        const T *c = (const T *)P.cost + (size_t)i * P.L;
        T *dc = TRAIN ? (T *)P.dcost + (size_t)i * P.L : nullptr;
        if (TRAIN && P.mask && P.mask[i] == 0) {
            if (P.dcost)
                for (int l = lane; l < P.L; l += 64) dc[l] = mrf_from_f32<T>(0.0f);
            if (lane == 0 && P.logp) P.logp[i] = 0.0f;
            continue;
        }
        float mn = INFINITY, s = 0.0f;
        for (int l = lane; l < P.L; l += 64) {
            const float v = mrf_to_f32(c[l]);
            if (v < mn) {
                s = s * mrf_exp_neg(v - mn) + 1.0f;
                mn = v;
            } else if (v < INFINITY || v != v) {
                s += mrf_exp_neg(mn - v);
            }
        }
        const float low = mrf_lanes_min<64>(mn);
        s = mrf_lanes_sum<64>(mn < INFINITY || s != s ? s * mrf_exp_neg(low - mn) : 0.0f);
        const int a = mrf_policy_label(P, i);
        const float ca = mrf_to_f32(c[a]);
        // (no label allowed: nothing is added, and the gradient is 0)
        const bool none = low == INFINITY && s == 0.0f;
        const float lp = none ? -INFINITY : (low - ca) - logf(s);
        if (lane == 0 && P.logp) P.logp[i] = lp;
        if constexpr (TRAIN) {
            float gain = 0.0f, div = 0.0f, slope = 0.0f;
            if (!none) mrf_policy_terms(P, i, lp, gain, div, slope);
            total_gain += (double)gain;
            total_div += (double)div;
            if (P.dcost) {
                const float g = slope * inv_n * P.scale, f = none ? 0.0f : g / s;
                for (int l = lane; l < P.L; l += 64) {
                    const float e = none ? 0.0f : mrf_exp_small(low - mrf_to_f32(c[l]));
                    dc[l] = mrf_from_f32<T>(f * e - (l == a ? g : 0.0f));
                }
            }
        }
    }
    if constexpr (TRAIN) {
        if (lane == 0) {
            sums[0][wv] = total_gain;
            sums[1][wv] = total_div;
        }
        __syncthreads();
        if (threadIdx.x < 2) {
            const double *w = sums[threadIdx.x];
            P.partial[2 * (size_t)blockIdx.x + threadIdx.x] = (w[0] + w[1]) + (w[2] + w[3]);
        }
    }
}

// the loss from the partial sums: one workgroup, the first 256 threads add every 256th of the first sum, the others of the second
__global__ void __launch_bounds__(512) mrf_policy_sum(const MrfPolicyParams P, int blocks, int count_blocks)
{
    __shared__ double waves[8];
    const long long n = mrf_policy_counted(P, count_blocks);
    const int which = threadIdx.x >> 8;
    double v = 0.0;
    for (int k = threadIdx.x & 255; k < blocks; k += 256) v += P.partial[2 * (size_t)k + which];
    v = mrf_wave_sum_f64(v);
    if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
    __syncthreads();
    if (threadIdx.x == 0) {
        const double gain = ((waves[0] + waves[1]) + (waves[2] + waves[3])) / (double)n;
        const double div = ((waves[4] + waves[5]) + (waves[6] + waves[7])) / (double)n;
        P.loss[0] = (float)(P.kl > 0.0f ? (double)P.kl * div - gain : -gain);
        P.loss[1] = (float)-gain;
        P.loss[2] = (float)div;
    }
}

using namespace mrf_host;

namespace {

int policy_check(int64_t N, int32_t L, int type, int label_bytes)
{
    if (N < 0 || N > 0x7fffffffLL) return MRF_ERR_BAD_SHAPE;
    if (label_bytes != 1 && label_bytes != 4) return MRF_ERR_BAD_ARGUMENT;
    if (L < 1 || (label_bytes == 1 && L > MRF_MAX_LABELS)) return MRF_ERR_BAD_LABELS;
    return known_type(type) ? MRF_OK : MRF_ERR_BAD_ARGUMENT;
}

template <class T> int logp_launch(const MrfPolicyParams &P, hipStream_t st)
{
    const long long rows = (P.N + 3) / 4;
    hipLaunchKernelGGL((mrf_policy_any<T, false>), dim3((unsigned)(rows < MRF_POLICY_BLOCKS ? rows : MRF_POLICY_BLOCKS)), dim3(256), 0, st, P, 0);
    return launch_status("mrf_softmin_logp");
}

template <class T> int policy_launch(const MrfPolicyParams &P, hipStream_t st)
{
    int counts = 0;
    if (P.mask) {
        const long long need = (P.N + 1023) / 1024;
        counts = (int)(need < MRF_POLICY_COUNTS ? need : MRF_POLICY_COUNTS);
        hipLaunchKernelGGL(mrf_policy_count, dim3((unsigned)counts), dim3(1024), 0, st, P);
        const int rc = launch_status("mrf_policy_count");
        if (rc != MRF_OK) return rc;
    }
    const long long rows = (P.N + 3) / 4;
    const int blocks = (int)(rows < MRF_POLICY_BLOCKS ? rows : MRF_POLICY_BLOCKS);
    hipLaunchKernelGGL((mrf_policy_any<T, true>), dim3((unsigned)blocks), dim3(256), 0, st, P, counts);
    const int rc = launch_status("mrf_policy");
    if (rc != MRF_OK) return rc;
    hipLaunchKernelGGL(mrf_policy_sum, dim3(1), dim3(512), 0, st, P, blocks, counts);
    return launch_status("mrf_policy_sum");
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
    const int rc = policy_check(n_pixels, L, cost_type, label_bytes);
    if (rc != MRF_OK) return rc;
    if (pixels_per_advantage < 1 || !(clip_low >= 0.0f) || !(clip_low < 1.0f) || !(clip_high >= 0.0f) || !(clip_high < INFINITY) ||
        !(kl_weight >= 0.0f) || !(kl_weight < INFINITY) || !(fabsf(grad_scale) < INFINITY))
        return MRF_ERR_BAD_ARGUMENT;
    if (!loss || !workspace || (n_pixels > 0 && (!cost || !labels || !advantage)) || (kl_weight > 0.0f && n_pixels > 0 && !ref_logp))
        return MRF_ERR_NULL_POINTER;
    if (workspace_bytes < mrf_softmin_policy_workspace_bytes()) return MRF_ERR_WORKSPACE_TOO_SMALL;
    MrfPolicyParams P = {};
    P.N = n_pixels; P.L = L; P.cost = cost; P.labels = labels; P.label_bytes = label_bytes; P.advantage = advantage;
    P.per = pixels_per_advantage; P.old_logp = old_logp; P.ref_logp = ref_logp; P.mask = mask; P.low = 1.0f - clip_low;
    P.high = 1.0f + clip_high; P.kl = kl_weight; P.scale = grad_scale; P.loss = loss; P.logp = logp; P.dcost = grad_cost;
    P.counts = (long long *)workspace;
    P.partial = (double *)((char *)workspace + sizeof(long long) * MRF_POLICY_COUNTS);
    hipStream_t st = (hipStream_t)hip_stream;
    if (n_pixels == 0) {
        P.mask = nullptr;
        hipLaunchKernelGGL(mrf_policy_sum, dim3(1), dim3(512), 0, st, P, 0, 0);
        return launch_status("mrf_policy_sum");
    }
    if (cost_type == MRF_F32) return policy_launch<float>(P, st);
    return cost_type == MRF_F16 ? policy_launch<mrf_f16>(P, st) : policy_launch<mrf_bf16>(P, st);
}

}  // extern "C"
