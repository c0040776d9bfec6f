// Layer normalisation over the channels of a pixel, forward and backward:
//   y = (x - mean) * rstd * gamma + beta,   mean, var over the C channels of a row, rstd = 1 / sqrt(var + eps)
//   t = dy * gamma,  xhat = (x - mean) * rstd,
//   dx = rstd * (t - mean_c(t) - xhat * mean_c(t * xhat)),   dgamma = sum_rows dy * xhat,   dbeta = sum_rows dy
//
// First form: one warp walks a row three times; the gradients of gamma and beta are summed by a second kernel, a thread per
// channel and range of rows, and joined in order by a third.
#include "common.cuh"

namespace dr {

__device__ __forceinline__ float ln_load(const float* p) { return *p; }
__device__ __forceinline__ float ln_load(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void ln_store(float* p, float v) { *p = v; }
__device__ __forceinline__ void ln_store(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

struct LnParams {
    size_t M;
    int C, ldx, ldy, lddx;      // ldy is dy's in the backward pass
    const void *x, *dy;
    void *y, *dx;
    const float *gamma, *beta, *mean_in, *rstd_in;
    float *mean, *rstd;
    float eps;
    float* partials;            // [n_part][2][C]
    int n_part;
    float *dgamma, *dbeta;
};

template <typename TI, typename TO>
__global__ void __launch_bounds__(256) ln_forward_kernel(const LnParams p) {
    const int lane = threadIdx.x & 31;
    for (size_t r = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5); r < p.M; r += (size_t)gridDim.x * 8) {
        const TI* x = (const TI*)p.x + r * p.ldx;
        TO* y = (TO*)p.y + r * p.ldy;
        float s = 0.f;
        for (int c = lane; c < p.C; c += 32) s += ln_load(x + c);
        const float mean = warp_sum(s) / (float)p.C;
        float q = 0.f;
        for (int c = lane; c < p.C; c += 32) {
            const float d = ln_load(x + c) - mean;
            q = fmaf(d, d, q);
        }
        const float rstd = 1.f / sqrtf(warp_sum(q) / (float)p.C + p.eps);
        for (int c = lane; c < p.C; c += 32) {
            const float h = (ln_load(x + c) - mean) * rstd;
            ln_store(y + c, fmaf(h, p.gamma ? p.gamma[c] : 1.f, p.beta ? p.beta[c] : 0.f));
        }
        if (lane == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
    }
}

template <typename TI, typename TO>
__global__ void __launch_bounds__(256) ln_backward_sums_kernel(const LnParams p) {
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= p.C) return;
    const size_t r0 = p.M * blockIdx.y / p.n_part, r1 = p.M * (blockIdx.y + 1) / p.n_part;
    float sg = 0.f, sb = 0.f;
    for (size_t r = r0; r < r1; ++r) {
        const float dy = ln_load((const TO*)p.dy + r * p.ldy + c);
        const float h = (ln_load((const TI*)p.x + r * p.ldx + c) - p.mean_in[r]) * p.rstd_in[r];
        sg = fmaf(dy, h, sg);
        sb += dy;
    }
    p.partials[(size_t)blockIdx.y * 2 * p.C + c] = sg;
    p.partials[(size_t)blockIdx.y * 2 * p.C + p.C + c] = sb;
}

__global__ void __launch_bounds__(256) ln_backward_join_kernel(const LnParams p) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= 2 * p.C) return;
    float* out = i < p.C ? p.dgamma : p.dbeta;
    if (!out) return;
    float s = 0.f;
    for (int k = 0; k < p.n_part; ++k) s += p.partials[(size_t)k * 2 * p.C + i];
    out[i < p.C ? i : i - p.C] = s;
}

template <typename TI, typename TO>
__global__ void __launch_bounds__(256) ln_backward_kernel(const LnParams p) {
    const int lane = threadIdx.x & 31;
    for (size_t r = (size_t)blockIdx.x * 8 + (threadIdx.x >> 5); r < p.M; r += (size_t)gridDim.x * 8) {
        const TI* x = (const TI*)p.x + r * p.ldx;
        const TO* dy = (const TO*)p.dy + r * p.ldy;
        TI* dx = (TI*)p.dx + r * p.lddx;
        const float mean = p.mean_in[r], rstd = p.rstd_in[r];
        float s1 = 0.f, s2 = 0.f;
        for (int c = lane; c < p.C; c += 32) {
            const float t = ln_load(dy + c) * (p.gamma ? p.gamma[c] : 1.f);
            s1 += t;
            s2 = fmaf(t, (ln_load(x + c) - mean) * rstd, s2);
        }
        s1 = warp_sum(s1) / (float)p.C;
        s2 = warp_sum(s2) / (float)p.C;
        for (int c = lane; c < p.C; c += 32) {
            const float t = ln_load(dy + c) * (p.gamma ? p.gamma[c] : 1.f);
            const float h = (ln_load(x + c) - mean) * rstd;
            ln_store(dx + c, rstd * (t - s1 - h * s2));
        }
    }
}

static int ln_parts(size_t M) {
    const size_t n = (M + 63) / 64;
    return (int)(n < 1 ? 1 : n > 512 ? 512 : n);
}

}  // namespace dr

using namespace dr;

#define LN_DISPATCH(KERNEL, GRID, P, FLAGS, STREAM)                                                                  \
    do {                                                                                                             \
        const bool xf = (FLAGS) & DR_LN_X_F32, yf = (FLAGS) & DR_LN_Y_F32;                                           \
        if (xf && yf) KERNEL<float, float><<<GRID, 256, 0, STREAM>>>(P);                                             \
        else if (xf) KERNEL<float, __nv_bfloat16><<<GRID, 256, 0, STREAM>>>(P);                                      \
        else if (yf) KERNEL<__nv_bfloat16, float><<<GRID, 256, 0, STREAM>>>(P);                                      \
        else KERNEL<__nv_bfloat16, __nv_bfloat16><<<GRID, 256, 0, STREAM>>>(P);                                      \
        count_launch();                                                                                              \
    } while (0)

static bool ln_aligned(const void* p, bool f32) { return ((uintptr_t)p & (f32 ? 3u : 1u)) == 0; }

extern "C" int dr_layernorm(size_t npix, int C, const void* x, int ldx, const float* gamma, const float* beta, float eps, void* y, int ldy,
                            float* mean, float* rstd, unsigned flags, void* stream) {
    if (!x || !y || C <= 0 || !(eps >= 0.f) || (flags & ~(unsigned)(DR_LN_X_F32 | DR_LN_Y_F32))) return DR_ERR_INVALID_ARG;
    if (ldx == 0) ldx = C;
    if (ldy == 0) ldy = C;
    if (ldx < C || ldy < C) return DR_ERR_INVALID_ARG;
    if (!ln_aligned(x, flags & DR_LN_X_F32) || !ln_aligned(y, flags & DR_LN_Y_F32) || !ln_aligned(gamma, true) || !ln_aligned(beta, true) ||
        !ln_aligned(mean, true) || !ln_aligned(rstd, true)) return DR_ERR_ALIGNMENT;
    if (npix == 0) return DR_OK;
    LnParams p = {};
    p.M = npix; p.C = C; p.x = x; p.ldx = ldx; p.gamma = gamma; p.beta = beta; p.eps = eps; p.y = y; p.ldy = ldy; p.mean = mean; p.rstd = rstd;
    const size_t blocks = (npix + 7) / 8, cap = (size_t)num_sms() * 8;
    LN_DISPATCH(ln_forward_kernel, (unsigned)(blocks < cap ? blocks : cap), p, flags, (cudaStream_t)stream);
    return launch_status();
}

extern "C" int dr_layernorm_bwd_workspace_bytes(size_t npix, int C, size_t* bytes) {
    if (!bytes || C <= 0) return DR_ERR_INVALID_ARG;
    *bytes = ((size_t)ln_parts(npix) * 2 * C * sizeof(float) + 255) / 256 * 256;
    return DR_OK;
}

extern "C" int dr_layernorm_bwd(size_t npix, int C, const void* dy, int lddy, const void* x, int ldx, const float* gamma, const float* mean,
                                const float* rstd, void* dx, int lddx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                                unsigned flags, void* stream) {
    if (!x || !dy || !dx || !mean || !rstd || C <= 0 || (flags & ~(unsigned)(DR_LN_X_F32 | DR_LN_Y_F32))) return DR_ERR_INVALID_ARG;
    if (lddy == 0) lddy = C;
    if (ldx == 0) ldx = C;
    if (lddx == 0) lddx = C;
    if (lddy < C || ldx < C || lddx < C) return DR_ERR_INVALID_ARG;
    const bool sums = dgamma || dbeta;
    if (sums && !workspace) return DR_ERR_INVALID_ARG;
    const bool xf = flags & DR_LN_X_F32, yf = flags & DR_LN_Y_F32;
    if (!ln_aligned(x, xf) || !ln_aligned(dx, xf) || !ln_aligned(dy, yf) || !ln_aligned(gamma, true) || !ln_aligned(mean, true) ||
        !ln_aligned(rstd, true) || !ln_aligned(dgamma, true) || !ln_aligned(dbeta, true) || (sums && ((uintptr_t)workspace & 255))) return DR_ERR_ALIGNMENT;
    size_t need = 0;
    dr_layernorm_bwd_workspace_bytes(npix, C, &need);
    if (sums && workspace_bytes < need) return DR_ERR_WORKSPACE;
    cudaStream_t s = (cudaStream_t)stream;
    if (npix == 0) {            // an empty sum
        if (dgamma && cudaMemsetAsync(dgamma, 0, (size_t)C * sizeof(float), s) != cudaSuccess) return DR_ERR_CUDA;
        if (dbeta && cudaMemsetAsync(dbeta, 0, (size_t)C * sizeof(float), s) != cudaSuccess) return DR_ERR_CUDA;
        return DR_OK;
    }
    LnParams p = {};
    p.M = npix; p.C = C; p.dy = dy; p.ldy = lddy; p.x = x; p.ldx = ldx; p.gamma = gamma; p.mean_in = mean; p.rstd_in = rstd; p.dx = dx; p.lddx = lddx;
    p.partials = (float*)workspace; p.n_part = ln_parts(npix); p.dgamma = dgamma; p.dbeta = dbeta;
    if (sums) {
        LN_DISPATCH(ln_backward_sums_kernel, dim3((unsigned)((C + 255) / 256), (unsigned)p.n_part), p, flags, s);
        int st = launch_status();
        if (st != DR_OK) return st;
        ln_backward_join_kernel<<<(unsigned)((2 * (size_t)C + 255) / 256), 256, 0, s>>>(p);
        count_launch();
        st = launch_status();
        if (st != DR_OK) return st;
    }
    const size_t blocks = (npix + 7) / 8, cap = (size_t)num_sms() * 8;
    LN_DISPATCH(ln_backward_kernel, (unsigned)(blocks < cap ? blocks : cap), p, flags, s);
    return launch_status();
}
