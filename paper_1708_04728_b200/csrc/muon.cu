// Orthogonalising an update by Newton-Schulz products, and the optimiser step that uses it:
//   X_0 = U / (|U|_F + eps),   A = X X^T,   X <- a X + (b A + c A A) X   (`steps` times),   O = X
//   v <- momentum v + g;  U = g + momentum v (Nesterov) or v;  w <- w - lr (sqrt(max(1, rows / cols)) O + decay w)
// X has n = min(rows, cols) rows: a taller U is worked on as its transpose.
//
// First form: everything in float32 on CUDA cores, a 64 x 64 tile of a product per block.
#include <cmath>

#include "common.cuh"

namespace dr {

constexpr int NS_NORM_BLOCKS = 128;

struct NsInput {
    int rows, cols, tall, n, m;
    const void* g;              // gradient (bf16 or f32), or the optimiser's float32 gradient
    int g_f32;
    float *v, *w;               // optimiser state, nullptr for the product alone
    float momentum;
    int nesterov;
    float eps;
};

__device__ __forceinline__ float ns_value(const NsInput& in, size_t i) {
    const float g = in.g_f32 ? ((const float*)in.g)[i] : __bfloat162float(((const __nv_bfloat16*)in.g)[i]);
    if (!in.v) return g;
    return in.nesterov ? fmaf(in.momentum, in.v[i], g) : in.v[i];
}

__global__ void __launch_bounds__(256) ns_momentum_kernel(const NsInput in, size_t n) {
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256)
        in.v[i] = fmaf(in.momentum, in.v[i], ((const float*)in.g)[i]);
}

__device__ double ns_block_sum(double s) {
    __shared__ double red[256];
    red[threadIdx.x] = s;
    __syncthreads();
    for (int o = 128; o; o >>= 1) {
        if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
        __syncthreads();
    }
    return red[0];
}

// sum of squares of matrix blockIdx.y, one partial per block
__global__ void __launch_bounds__(256) ns_norm_kernel(const NsInput in, double* partial) {
    const size_t per = (size_t)in.rows * in.cols;
    double s = 0.;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (size_t)NS_NORM_BLOCKS * 256) {
        const double u = ns_value(in, blockIdx.y * per + i);
        s += u * u;
    }
    s = ns_block_sum(s);
    if (threadIdx.x == 0) partial[(size_t)blockIdx.y * NS_NORM_BLOCKS + blockIdx.x] = s;
}

__global__ void __launch_bounds__(256) ns_scale_kernel(const NsInput in, const double* partial, float* X) {
    const double s = ns_block_sum(threadIdx.x < NS_NORM_BLOCKS ? partial[(size_t)blockIdx.y * NS_NORM_BLOCKS + threadIdx.x] : 0.);
    const float inv = (float)(1. / (sqrt(s) + (double)in.eps));
    const size_t per = (size_t)in.rows * in.cols;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (size_t)gridDim.x * 256) {
        const size_t r = i / in.cols, c = i - r * in.cols;
        X[blockIdx.y * per + (in.tall ? c * in.rows + r : i)] = ns_value(in, blockIdx.y * per + i) * inv;
    }
}

// out[i][j] = alpha * add[i][j] + beta * sum_k P[i][k] * (TRANS ? Q[j][k] : Q[k][j])
template <bool TRANS>
__global__ void __launch_bounds__(256) ns_product_kernel(int I, int J, int K, const float* P, const float* Q, float alpha, const float* add, float beta, float* out) {
    __shared__ float sp[16][65], sq[16][65];
    P += (size_t)blockIdx.z * I * K;
    Q += (size_t)blockIdx.z * J * K;
    const size_t o = (size_t)blockIdx.z * I * J;
    const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, ti = threadIdx.x >> 4, tj = threadIdx.x & 15;
    float acc[4][4] = {};
    for (int k0 = 0; k0 < K; k0 += 16) {
        for (int e = threadIdx.x; e < 1024; e += 256) {
            const int i = e >> 4, k = e & 15;
            sp[k][i] = i0 + i < I && k0 + k < K ? P[(size_t)(i0 + i) * K + k0 + k] : 0.f;
            if (TRANS) sq[k][i] = j0 + i < J && k0 + k < K ? Q[(size_t)(j0 + i) * K + k0 + k] : 0.f;
            const int kk = e >> 6, j = e & 63;
            if (!TRANS) sq[kk][j] = j0 + j < J && k0 + kk < K ? Q[(size_t)(k0 + kk) * J + j0 + j] : 0.f;
        }
        __syncthreads();
        for (int k = 0; k < 16; ++k)
            for (int a = 0; a < 4; ++a)
                for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(sp[k][ti + 16 * a], sq[k][tj + 16 * b], acc[a][b]);
        __syncthreads();
    }
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int i = i0 + ti + 16 * a, j = j0 + tj + 16 * b;
            if (i < I && j < J) {
                const size_t e = o + (size_t)i * J + j;
                out[e] = beta * acc[a][b] + (add ? alpha * add[e] : 0.f);
            }
        }
}

__global__ void __launch_bounds__(256) ns_finish_kernel(const NsInput in, const float* X, float lr_scale, float keep, __nv_bfloat16* out) {
    const size_t per = (size_t)in.rows * in.cols;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < per; i += (size_t)gridDim.x * 256) {
        const size_t r = i / in.cols, c = i - r * in.cols, e = blockIdx.y * per + i;
        const float x = X[blockIdx.y * per + (in.tall ? c * in.rows + r : i)];
        if (in.w) {
            const float wn = fmaf(-lr_scale, x, keep * in.w[e]);
            in.w[e] = wn;
            if (out) out[e] = __float2bfloat16_rn(wn);
        } else {
            out[e] = __float2bfloat16_rn(x);
        }
    }
}

struct NsWorkspace { size_t partial, x0, x1, a, b, total; };
static NsWorkspace ns_workspace(int batch, int rows, int cols) {
    const size_t n = rows < cols ? rows : cols, x = (size_t)batch * rows * cols * sizeof(float), a = (size_t)batch * n * n * sizeof(float);
    auto up = [](size_t b) { return (b + 255) / 256 * 256; };
    NsWorkspace w;
    w.partial = 0;
    w.x0 = up((size_t)batch * NS_NORM_BLOCKS * sizeof(double));
    w.x1 = w.x0 + up(x);
    w.a = w.x1 + up(x);
    w.b = w.a + up(a);
    w.total = w.b + up(a);
    return w;
}

static int ns_check(int batch, int rows, int cols, int steps, const float* coef, float eps) {
    if (batch < 0 || rows <= 0 || cols <= 0 || steps < 1 || !(eps >= 0.f)) return DR_ERR_INVALID_ARG;
    if (rows > DR_NS_MAX_DIM || cols > DR_NS_MAX_DIM || steps > DR_NS_MAX_STEPS || batch > 65535) return DR_ERR_UNSUPPORTED;
    if (coef)
        for (int i = 0; i < 3 * steps; ++i)
            if (!std::isfinite(coef[i])) return DR_ERR_INVALID_ARG;
    return DR_OK;
}

static int ns_run(int batch, const NsInput& in, int steps, const float* coef, float lr_scale, float keep, __nv_bfloat16* out, char* ws, cudaStream_t s) {
    const NsWorkspace l = ns_workspace(batch, in.rows, in.cols);
    const size_t per = (size_t)in.rows * in.cols;
    const unsigned eb = (unsigned)std::min<size_t>((per + 255) / 256, (size_t)num_sms() * 8);
    double* partial = (double*)(ws + l.partial);
    float *X = (float*)(ws + l.x0), *Y = (float*)(ws + l.x1), *A = (float*)(ws + l.a), *B = (float*)(ws + l.b);
    if (in.v) {
        ns_momentum_kernel<<<(unsigned)num_sms() * 8, 256, 0, s>>>(in, per * batch);
        count_launch();
    }
    ns_norm_kernel<<<dim3(NS_NORM_BLOCKS, batch), 256, 0, s>>>(in, partial);
    ns_scale_kernel<<<dim3(eb, batch), 256, 0, s>>>(in, partial, X);
    const unsigned tn = (in.n + 63) / 64, tm = (in.m + 63) / 64;
    for (int k = 0; k < steps; ++k) {
        const float a = coef ? coef[3 * k] : 3.4445f, b = coef ? coef[3 * k + 1] : -4.7750f, c = coef ? coef[3 * k + 2] : 2.0315f;
        ns_product_kernel<true><<<dim3(tn, tn, batch), 256, 0, s>>>(in.n, in.n, in.m, X, X, 0.f, nullptr, 1.f, A);
        ns_product_kernel<false><<<dim3(tn, tn, batch), 256, 0, s>>>(in.n, in.n, in.n, A, A, b, A, c, B);
        ns_product_kernel<false><<<dim3(tm, tn, batch), 256, 0, s>>>(in.n, in.m, in.n, B, X, a, X, 1.f, Y);
        std::swap(X, Y);
    }
    ns_finish_kernel<<<dim3(eb, batch), 256, 0, s>>>(in, X, lr_scale, keep, out);
    count_launch(3 + 3 * steps);
    return launch_status();
}

}  // namespace dr

using namespace dr;

extern "C" int dr_orthogonalise_workspace_bytes(int batch, int rows, int cols, size_t* bytes) {
    if (!bytes) return DR_ERR_INVALID_ARG;
    const int st = ns_check(batch, rows, cols, 1, nullptr, 0.f);
    if (st != DR_OK) return st;
    *bytes = ns_workspace(batch, rows, cols).total;
    return DR_OK;
}

extern "C" int dr_orthogonalise(int batch, int rows, int cols, const void* g, int steps, const float* coef, float eps, void* o, void* workspace,
                                size_t workspace_bytes, unsigned flags, void* stream) {
    const int st = ns_check(batch, rows, cols, steps, coef, eps);
    if (st != DR_OK) return st;
    if (!g || !o || !workspace || (flags & ~(unsigned)DR_NS_G_F32)) return DR_ERR_INVALID_ARG;
    const bool f32 = flags & DR_NS_G_F32;
    if (((uintptr_t)g & (f32 ? 3u : 1u)) || ((uintptr_t)o & 1u) || ((uintptr_t)workspace & 255)) return DR_ERR_ALIGNMENT;
    if (workspace_bytes < ns_workspace(batch, rows, cols).total) return DR_ERR_WORKSPACE;
    if (batch == 0) return DR_OK;
    NsInput in = {};
    in.rows = rows; in.cols = cols; in.tall = rows > cols; in.n = in.tall ? cols : rows; in.m = in.tall ? rows : cols;
    in.g = g; in.g_f32 = f32; in.eps = eps;
    return ns_run(batch, in, steps, coef, 0.f, 0.f, (__nv_bfloat16*)o, (char*)workspace, (cudaStream_t)stream);
}

extern "C" int dr_muon_update(int batch, int rows, int cols, float* w, float* v, const float* g, float lr, float momentum, float decay, int nesterov,
                              int steps, const float* coef, float eps, void* w_bf16, void* workspace, size_t workspace_bytes, void* stream) {
    const int st = ns_check(batch, rows, cols, steps, coef, eps);
    if (st != DR_OK) return st;
    if (!w || !v || !g || !workspace) return DR_ERR_INVALID_ARG;
    if (((uintptr_t)w & 3u) || ((uintptr_t)v & 3u) || ((uintptr_t)g & 3u) || ((uintptr_t)w_bf16 & 1u) || ((uintptr_t)workspace & 255)) return DR_ERR_ALIGNMENT;
    if (workspace_bytes < ns_workspace(batch, rows, cols).total) return DR_ERR_WORKSPACE;
    if (batch == 0) return DR_OK;
    NsInput in = {};
    in.rows = rows; in.cols = cols; in.tall = rows > cols; in.n = in.tall ? cols : rows; in.m = in.tall ? rows : cols;
    in.g = g; in.g_f32 = 1; in.eps = eps; in.v = v; in.w = w; in.momentum = momentum; in.nesterov = nesterov != 0;
    const float scale = rows > cols ? sqrtf((float)rows / (float)cols) : 1.f;
    return ns_run(batch, in, steps, coef, lr * scale, 1.f - lr * decay, (__nv_bfloat16*)w_bf16, (char*)workspace, (cudaStream_t)stream);
}
