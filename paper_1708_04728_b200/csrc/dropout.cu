// Dropout: y = residual + keep * x / (1 - p), the mask drawn by a counter-based generator (dropout.cuh) and never stored; the backward
// pass is the same call on the gradient.
#include <climits>

#include "common.cuh"
#include "dropout.cuh"

namespace dr {

struct DropParams {
    unsigned long long n;       // elements
    int C, ldx, ldr, ldy;
    const void *x, *r;
    void* y;
    DropKey key;
};

template <typename T> __device__ __forceinline__ float drop_ld(const void* p, size_t i);
template <> __device__ __forceinline__ float drop_ld<float>(const void* p, size_t i) { return ((const float*)p)[i]; }
template <> __device__ __forceinline__ float drop_ld<__nv_bfloat16>(const void* p, size_t i) { return __bfloat162float(((const __nv_bfloat16*)p)[i]); }
__device__ __forceinline__ void drop_st(float* p, float v) { *p = v; }
__device__ __forceinline__ void drop_st(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

template <typename TX, typename TY>
__global__ void __launch_bounds__(256) dropout_kernel(const DropParams p) {
    const unsigned long long off = drop_offset(p.key);
    for (unsigned long long e = (unsigned long long)blockIdx.x * blockDim.x + threadIdx.x; e < p.n; e += (unsigned long long)gridDim.x * blockDim.x) {
        const size_t row = e / p.C;
        const int col = (int)(e - row * p.C);
        const float v = drop_keep_at(p.key, off, e) ? drop_ld<TX>(p.x, row * p.ldx + col) * p.key.scale : 0.f;
        drop_st((TY*)p.y + row * p.ldy + col, p.r ? drop_ld<TY>(p.r, row * p.ldr + col) + v : v);
    }
}

static bool type_aligned(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }

}  // namespace dr

using namespace dr;

extern "C" int dr_dropout(size_t rows, int C, const void* x, int ldx, const void* residual, int ldr, void* y, int ldy, double p, unsigned long long seed,
                          unsigned long long offset, const unsigned long long* step, unsigned flags, void* stream) {
    if (C <= 0 || (flags & ~(DR_DROP_X_F32 | DR_DROP_Y_F32)) || !drop_p_ok(p)) return DR_ERR_INVALID_ARG;
    if (!ldx) ldx = C;
    if (!ldr) ldr = C;
    if (!ldy) ldy = C;
    if (ldx < C || ldr < C || ldy < C || rows > (size_t)LLONG_MAX / 16 / C) return DR_ERR_INVALID_ARG;
    if (rows == 0) return DR_OK;
    if (!x || !y) return DR_ERR_INVALID_ARG;
    const bool xf = flags & DR_DROP_X_F32, yf = flags & DR_DROP_Y_F32;
    if (!type_aligned(x, xf ? 4 : 2) || !type_aligned(y, yf ? 4 : 2) || !type_aligned(residual, yf ? 4 : 2) || !type_aligned(step, 8)) return DR_ERR_ALIGNMENT;
    DropParams q;
    q.n = (unsigned long long)rows * C;
    q.C = C; q.ldx = ldx; q.ldr = ldr; q.ldy = ldy;
    q.x = x; q.r = residual; q.y = y;
    q.key = drop_key(p, seed, offset, step);
    const unsigned long long want = (q.n + 255) / 256, most = (unsigned long long)num_sms() * 8;
    const int grid = (int)(want < most ? want : most);
    const cudaStream_t s = (cudaStream_t)stream;
    if (xf && yf) dropout_kernel<float, float><<<grid, 256, 0, s>>>(q);
    else if (xf) dropout_kernel<float, __nv_bfloat16><<<grid, 256, 0, s>>>(q);
    else if (yf) dropout_kernel<__nv_bfloat16, float><<<grid, 256, 0, s>>>(q);
    else dropout_kernel<__nv_bfloat16, __nv_bfloat16><<<grid, 256, 0, s>>>(q);
    count_launch();
    return launch_status();
}
