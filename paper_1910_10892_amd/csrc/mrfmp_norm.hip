// Layer norm over the rows of a matrix, forward and backward (see mrf_layer_norm_forward in the header for the formulas).
#include "mrfmp_learn.h"

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

// ---- a wavefront per row: any length, any alignment
template <class X, class Y>
__global__ void __launch_bounds__(256) mrf_norm_fwd_any(const MrfNormParams Q)
{
    const int lane = threadIdx.x & 63;
    const long long step = (long long)gridDim.x * 4;
    const float inv = 1.0f / (float)Q.C;
    for (long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); r < Q.N; r += step) {
        const X *x = (const X *)Q.x + (size_t)r * Q.C;
        Y *y = (Y *)Q.y + (size_t)r * Q.C;
        float s = 0.0f;
        for (int c = lane; c < Q.C; c += 64) s += mrf_to_f32(x[c]);
        const float mu = mrf_lanes_sum<64>(s) * inv;
        s = 0.0f;
        for (int c = lane; c < Q.C; c += 64) {
            const float d = mrf_to_f32(x[c]) - mu;
            s += d * d;
        }
        const float rs = 1.0f / sqrtf(mrf_lanes_sum<64>(s) * inv + Q.eps);
        for (int c = lane; c < Q.C; c += 64) {
            const float h = (mrf_to_f32(x[c]) - mu) * rs;
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
    const float inv = 1.0f / (float)Q.C;
    for (long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); r < Q.N; r += step) {
        const X *x = (const X *)Q.x + (size_t)r * Q.C;
        const Y *dy = (const Y *)Q.dy + (size_t)r * Q.C;
        X *dx = (X *)Q.dx + (size_t)r * Q.C;
        const float mu = Q.mean[r], rs = Q.rstd[r];
        float sa = 0.0f, sh = 0.0f;
        for (int c = lane; c < Q.C; c += 64) {
            const float h = (mrf_to_f32(x[c]) - mu) * rs;
            const float a = mrf_to_f32(dy[c]) * (Q.gamma ? Q.gamma[c] : 1.0f);
            sa += a;
            sh = fmaf(a, h, sh);
        }
        sa = mrf_lanes_sum<64>(sa) * inv;
        sh = mrf_lanes_sum<64>(sh) * inv;
        for (int c = lane; c < Q.C; c += 64) {
            const float h = (mrf_to_f32(x[c]) - mu) * rs;
            const float a = mrf_to_f32(dy[c]) * (Q.gamma ? Q.gamma[c] : 1.0f);
            dx[c] = mrf_from_f32<X>(rs * (a - sa - h * sh));
        }
    }
}

// sums over rows: grid (columns / 64, P), lane = column, a workgroup takes every P-th run of four rows
template <class X, class Y>
__global__ void __launch_bounds__(256) mrf_norm_param_any(const MrfNormParams Q)
{
    __shared__ float sums[2][4][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const int c = blockIdx.x * 64 + lane;
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
}

// weight and bias gradients from the P partial sums of a column, in order; grid (2 C / 64), 16 wavefronts share the partials
__global__ void __launch_bounds__(1024) mrf_norm_param_sum(const MrfNormParams Q)
{
    __shared__ float sums[16][64];
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const long long c = (long long)blockIdx.x * 64 + lane;      // [0, C) weight, [C, 2 C) bias
    float s = 0.0f;
    if (c < 2LL * Q.C)
        for (int p = wv; p < Q.P; p += 16) s += Q.partial[(size_t)p * 2 * Q.C + c];
    sums[wv][lane] = s;
    __syncthreads();
    if (wv == 0 && c < 2LL * Q.C) {
        s = 0.0f;
        for (int w = 0; w < 16; ++w) s += sums[w][lane];
        if (c < Q.C) {
            if (Q.dgamma) Q.dgamma[c] = s;
        } else if (Q.dbeta) {
            Q.dbeta[c - Q.C] = s;
        }
    }
}

using namespace mrf_host;

namespace {

// partial sums of the weight's gradient: no more than rows in fours, 8 MiB of them for rows of up to 16,384
int norm_partials(int64_t n_rows, int32_t C)
{
    long long p = (1LL << 20) / C;
    p = p < 64 ? 64 : (p > 1024 ? 1024 : p);
    const long long rows = (n_rows + 3) / 4;
    return (int)(p < rows ? p : rows);
}

int norm_check(int64_t n_rows, int32_t C, int x_type, int y_type)
{
    if (n_rows < 0 || n_rows > 0x7fffffffLL || C < 1) return MRF_ERR_BAD_SHAPE;
    if (!known_type(x_type) || !known_type(y_type) || (y_type != x_type && y_type != MRF_F32)) return MRF_ERR_BAD_ARGUMENT;
    return MRF_OK;
}

template <class X, class Y> int norm_forward(const MrfNormParams &Q, hipStream_t st)
{
    const long long rows = (Q.N + 3) / 4;
    hipLaunchKernelGGL((mrf_norm_fwd_any<X, Y>), dim3((unsigned)(rows < 8192 ? rows : 8192)), dim3(256), 0, st, Q);
    return launch_status("mrf_norm_fwd");
}

template <class X, class Y> int norm_backward(const MrfNormParams &Q, hipStream_t st)
{
    const long long rows = (Q.N + 3) / 4;
    if (Q.N > 0 && Q.dx) {
        hipLaunchKernelGGL((mrf_norm_bwd_any<X, Y>), dim3((unsigned)(rows < 8192 ? rows : 8192)), dim3(256), 0, st, Q);
        const int rc = launch_status("mrf_norm_bwd");
        if (rc != MRF_OK) return rc;
    }
    if (!Q.dgamma && !Q.dbeta) return MRF_OK;
    if (Q.N > 0) {
        hipLaunchKernelGGL((mrf_norm_param_any<X, Y>), dim3((unsigned)((Q.C + 63) / 64), (unsigned)Q.P), dim3(256), 0, st, Q);
        const int rc = launch_status("mrf_norm_param");
        if (rc != MRF_OK) return rc;
    }
    hipLaunchKernelGGL(mrf_norm_param_sum, dim3((unsigned)((2LL * Q.C + 63) / 64)), dim3(1024), 0, st, Q);
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
