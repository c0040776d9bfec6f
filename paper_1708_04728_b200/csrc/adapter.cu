// A 1 x 1 (or fully connected) layer with the low-rank adapters of many requests beside its shared filters, forward and backward:
//   t = D(x) A_a^T,  y = act(x W^T + bias + scale_a t B_a^T);     u = scale_a dy B_a,  dx = dy W + D(u A_a),  dA_a = sum u^T D(x),
//   dB_a = scale_a sum dy^T t,     a the adapter of the request that a row belongs to, D the dropout of dropout.cuh.
#include <climits>

#include "common.cuh"
#include "dropout.cuh"

namespace dr {

constexpr int ROW_SHARED = -1;      // a row of a request without an adapter
constexpr int ROW_NONE = -2;        // a row of no request: left as it was

struct AdRows {
    int M, segments, adapters;
    const int *row_start, *adapter;
};

// The adapter of row m.  Whatever the offsets hold, the search stays inside them; an adapter out of range is none.
__device__ __forceinline__ int adapter_of_row(const AdRows& r, int m) {
    int lo = 0, hi = r.segments + 1;            // number of offsets <= m
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (r.row_start[mid] <= m) lo = mid + 1;
        else hi = mid;
    }
    if (lo == 0 || lo > r.segments) return ROW_NONE;
    const int a = r.adapter[lo - 1];
    return a >= 0 && a < r.adapters ? a : ROW_SHARED;
}

__global__ void adapter_rows_kernel(const AdRows r, int* __restrict__ row_id) {
    const int m = blockIdx.x * blockDim.x + threadIdx.x;
    if (m < r.M) row_id[m] = r.segments > 0 ? adapter_of_row(r, m) : ROW_NONE;
}

// out[m][r] = factor * sum_k D(z)[m][k] f_a[r][k], f_a rows of K (fr = K, fk = 1) or columns (fr = 1, fk = R)
__global__ void adapter_down_kernel(int M, int K, int R, const __nv_bfloat16* __restrict__ z, int ldz, const __nv_bfloat16* __restrict__ f, int fr, int fk,
                                    const float* __restrict__ scale, const DropKey key, const int* __restrict__ row_id, float* __restrict__ out, float* __restrict__ keep) {
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (size_t)M * R) return;
    const int m = (int)(i / R), r = (int)(i - (size_t)m * R), a = row_id[m];
    float s = 0.f;
    if (a >= 0) {
        const unsigned long long off = drop_offset(key);
        const __nv_bfloat16* w = f + (size_t)a * R * K + (size_t)r * fr;
        for (int k = 0; k < K; ++k) {
            const bool kept = key.thr == 0 || drop_keep_at(key, off, (unsigned long long)m * K + k);
            if (kept) s = fmaf(__bfloat162float(z[(size_t)m * ldz + k]), __bfloat162float(w[(size_t)k * fk]), s);
        }
        s *= key.thr ? key.scale : 1.f;
        if (scale) s *= scale[a];
    }
    out[i] = s;
    if (keep && a != ROW_NONE) keep[i] = s;
}

__global__ void adapter_forward_kernel(int M, int K, int N, int R, const __nv_bfloat16* __restrict__ x, int ldx, const __nv_bfloat16* __restrict__ w,
                                       const float* __restrict__ bias, const __nv_bfloat16* __restrict__ b, const float* __restrict__ scale,
                                       const int* __restrict__ row_id, const float* __restrict__ t, unsigned flags, void* __restrict__ y, int ldy) {
    const int n = blockIdx.x * blockDim.x + threadIdx.x, m = blockIdx.y + blockIdx.z * 32768;
    if (n >= N || m >= M || row_id[m] == ROW_NONE) return;
    float s = 0.f, l = 0.f;
    for (int k = 0; k < K; ++k) s = fmaf(__bfloat162float(x[(size_t)m * ldx + k]), __bfloat162float(w[(size_t)n * K + k]), s);
    const int a = row_id[m];
    if (a >= 0) {
        for (int r = 0; r < R; ++r) l = fmaf(t[(size_t)m * R + r], __bfloat162float(b[((size_t)a * N + n) * R + r]), l);
        s = fmaf(scale ? scale[a] : 1.f, l, s);
    }
    if (flags & DR_BIAS) s += bias[n];
    if (flags & DR_RELU) s = s < 0.f ? 0.f : s;         // NaN stays NaN
    if (flags & DR_OUT_F32) ((float*)y)[(size_t)m * ldy + n] = s;
    else ((__nv_bfloat16*)y)[(size_t)m * ldy + n] = __float2bfloat16_rn(s);
}

__global__ void adapter_dx_kernel(int M, int K, int N, int R, const __nv_bfloat16* __restrict__ dy, int lddy, const __nv_bfloat16* __restrict__ w,
                                  const __nv_bfloat16* __restrict__ f, const int* __restrict__ row_id, const float* __restrict__ u, const DropKey key,
                                  __nv_bfloat16* __restrict__ dx, int lddx) {
    const int k = blockIdx.x * blockDim.x + threadIdx.x, m = blockIdx.y + blockIdx.z * 32768;
    if (k >= K || m >= M || row_id[m] == ROW_NONE) return;
    float s = 0.f, l = 0.f;
    for (int n = 0; n < N; ++n) s = fmaf(__bfloat162float(dy[(size_t)m * lddy + n]), __bfloat162float(w[(size_t)n * K + k]), s);
    const int a = row_id[m];
    if (a >= 0) {
        for (int r = 0; r < R; ++r) l = fmaf(u[(size_t)m * R + r], __bfloat162float(f[((size_t)a * R + r) * K + k]), l);
        if (key.thr == 0) s += l;
        else if (drop_keep_at(key, drop_offset(key), (unsigned long long)m * K + k)) s = fmaf(key.scale, l, s);
    }
    dx[(size_t)m * lddx + k] = __float2bfloat16_rn(s);
}

// out[a][r][c] (rc) or out[a][c][r]: sum over the rows of adapter a of factor * p[m][r] * D(z)[m][c]
__global__ void adapter_grad_kernel(int M, int C, int R, int adapters, const __nv_bfloat16* __restrict__ z, int ldz, const float* __restrict__ p,
                                    const float* __restrict__ scale, const int* __restrict__ row_id, const DropKey key, int rc, float* __restrict__ out) {
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i >= (size_t)adapters * R * C) return;
    const int a = (int)(i / ((size_t)R * C));
    const int rest = (int)(i - (size_t)a * R * C);
    const int r = rc ? rest / C : rest % R, c = rc ? rest % C : rest / R;
    const unsigned long long off = drop_offset(key);
    float s = 0.f;
    for (int m = 0; m < M; ++m)
        if (row_id[m] == a && (key.thr == 0 || drop_keep_at(key, off, (unsigned long long)m * C + c)))
            s = fmaf(p[(size_t)m * R + r], __bfloat162float(z[(size_t)m * ldz + c]), s);
    if (key.thr) s *= key.scale;
    out[i] = scale ? s * scale[a] : s;
}

static size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

static int desc_check(const dr_adapter_desc* d, int M) {
    if (!d || d->Cin <= 0 || d->Cout <= 0 || d->rank <= 0 || d->adapters <= 0 || M < 0) return DR_ERR_INVALID_ARG;
    if ((d->flags & ~(DR_BIAS | DR_RELU | DR_OUT_F32)) || !drop_p_ok(d->drop_p)) return DR_ERR_INVALID_ARG;
    if (d->rank > DR_ADAPTER_MAX_RANK || d->Cin > DR_ADAPTER_MAX_CHANNELS || d->Cout > DR_ADAPTER_MAX_CHANNELS || d->adapters > DR_ADAPTER_MAX_ADAPTERS ||
        M > DR_ADAPTER_MAX_ROWS)
        return DR_ERR_UNSUPPORTED;
    return DR_OK;
}
static int ld_check(int* ld, int C) {
    if (!*ld) *ld = C;
    return *ld < C ? DR_ERR_INVALID_ARG : DR_OK;
}

}  // namespace dr

using namespace dr;

extern "C" int dr_adapter_workspace_bytes(const dr_adapter_desc* d, int M, int ldx, size_t* bytes) {
    const int rc = desc_check(d, M);
    if (rc != DR_OK) return rc;
    if (!bytes || ld_check(&ldx, d->Cin) != DR_OK) return DR_ERR_INVALID_ARG;
    *bytes = up256((size_t)M * 4) + up256((size_t)M * d->rank * 4);
    return DR_OK;
}

extern "C" int dr_adapter_bwd_workspace_bytes(const dr_adapter_desc* d, int M, int ldx, int lddy, size_t* bytes) {
    const int rc = desc_check(d, M);
    if (rc != DR_OK) return rc;
    if (!bytes || ld_check(&ldx, d->Cin) != DR_OK || ld_check(&lddy, d->Cout) != DR_OK) return DR_ERR_INVALID_ARG;
    *bytes = up256((size_t)M * 4) + up256((size_t)M * d->rank * 4);
    return DR_OK;
}

extern "C" int dr_adapter(const dr_adapter_desc* d, int M, const void* x, int ldx, const void* w, const float* bias, const void* a, const void* b,
                          const float* scale, int segments, const int* row_start, const int* adapter, void* y, int ldy, float* t,
                          const unsigned long long* step, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = desc_check(d, M);
    if (rc != DR_OK) return rc;
    if (ld_check(&ldx, d->Cin) != DR_OK || ld_check(&ldy, d->Cout) != DR_OK || segments < 0) return DR_ERR_INVALID_ARG;
    if (M == 0 || segments == 0) return DR_OK;
    if (!x || !w || !a || !b || !y || !row_start || !adapter || !workspace || ((d->flags & DR_BIAS) && !bias)) return DR_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(w) || !aligned16(a) || !aligned16(b) || ((uintptr_t)y & ((d->flags & DR_OUT_F32) ? 3 : 1)) || ((uintptr_t)bias & 3) ||
        ((uintptr_t)scale & 3) || ((uintptr_t)row_start & 3) || ((uintptr_t)adapter & 3) || ((uintptr_t)t & 3) || ((uintptr_t)step & 7) ||
        ((uintptr_t)workspace & 255))
        return DR_ERR_ALIGNMENT;
    size_t need = 0;
    rc = dr_adapter_workspace_bytes(d, M, ldx, &need);
    if (rc != DR_OK) return rc;
    if (workspace_bytes < need) return DR_ERR_WORKSPACE;
    const cudaStream_t s = (cudaStream_t)stream;
    const int K = d->Cin, N = d->Cout, R = d->rank;
    int* row_id = (int*)workspace;
    float* tw = (float*)((char*)workspace + up256((size_t)M * 4));
    const AdRows rows = {M, segments, d->adapters, row_start, adapter};
    const DropKey key = drop_key(d->drop_p, d->drop_seed, d->drop_offset, step);
    adapter_rows_kernel<<<(M + 255) / 256, 256, 0, s>>>(rows, row_id);
    adapter_down_kernel<<<(unsigned)(((size_t)M * R + 255) / 256), 256, 0, s>>>(M, K, R, (const __nv_bfloat16*)x, ldx, (const __nv_bfloat16*)a, K, 1, nullptr, key, row_id, tw, t);
    adapter_forward_kernel<<<dim3((N + 127) / 128, M < 32768 ? M : 32768, (M + 32767) / 32768), 128, 0, s>>>(
        M, K, N, R, (const __nv_bfloat16*)x, ldx, (const __nv_bfloat16*)w, bias, (const __nv_bfloat16*)b, scale, row_id, tw, d->flags, y, ldy);
    count_launch(3);
    return launch_status();
}

extern "C" int dr_adapter_bwd(const dr_adapter_desc* d, int M, const void* dy, int lddy, const void* x, int ldx, const void* w, const void* a, const void* b,
                              const float* scale, int segments, const int* row_start, const int* adapter, const float* t, void* dx, int lddx, float* da,
                              float* db, const unsigned long long* step, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = desc_check(d, M);
    if (rc != DR_OK) return rc;
    if (ld_check(&ldx, d->Cin) != DR_OK || ld_check(&lddx, d->Cin) != DR_OK || ld_check(&lddy, d->Cout) != DR_OK || segments < 0) return DR_ERR_INVALID_ARG;
    if (((uintptr_t)da & 3) || ((uintptr_t)db & 3)) return DR_ERR_ALIGNMENT;
    const cudaStream_t s = (cudaStream_t)stream;
    const int K = d->Cin, N = d->Cout, R = d->rank;
    if (M == 0 || segments == 0) {
        if (da && cudaMemsetAsync(da, 0, (size_t)d->adapters * R * K * 4, s) != cudaSuccess) return DR_ERR_CUDA;
        if (db && cudaMemsetAsync(db, 0, (size_t)d->adapters * R * N * 4, s) != cudaSuccess) return DR_ERR_CUDA;
        return DR_OK;
    }
    if (!dy || !w || !a || !b || !row_start || !adapter || !workspace || (da && !x) || (db && !t)) return DR_ERR_INVALID_ARG;
    if (!aligned16(dy) || !aligned16(x) || !aligned16(w) || !aligned16(a) || !aligned16(b) || ((uintptr_t)dx & 1) || ((uintptr_t)scale & 3) ||
        ((uintptr_t)row_start & 3) || ((uintptr_t)adapter & 3) || ((uintptr_t)t & 3) || ((uintptr_t)step & 7) || ((uintptr_t)workspace & 255))
        return DR_ERR_ALIGNMENT;
    size_t need = 0;
    rc = dr_adapter_bwd_workspace_bytes(d, M, ldx, lddy, &need);
    if (rc != DR_OK) return rc;
    if (workspace_bytes < need) return DR_ERR_WORKSPACE;
    int* row_id = (int*)workspace;
    float* u = (float*)((char*)workspace + up256((size_t)M * 4));
    const AdRows rows = {M, segments, d->adapters, row_start, adapter};
    const DropKey key = drop_key(d->drop_p, d->drop_seed, d->drop_offset, step), none = drop_key(0., 0, 0, nullptr);
    adapter_rows_kernel<<<(M + 255) / 256, 256, 0, s>>>(rows, row_id);
    adapter_down_kernel<<<(unsigned)(((size_t)M * R + 255) / 256), 256, 0, s>>>(M, N, R, (const __nv_bfloat16*)dy, lddy, (const __nv_bfloat16*)b, 1, R, scale, none, row_id, u, nullptr);
    count_launch(2);
    if (dx) {
        adapter_dx_kernel<<<dim3((K + 127) / 128, M < 32768 ? M : 32768, (M + 32767) / 32768), 128, 0, s>>>(
            M, K, N, R, (const __nv_bfloat16*)dy, lddy, (const __nv_bfloat16*)w, (const __nv_bfloat16*)a, row_id, u, key, (__nv_bfloat16*)dx, lddx);
        count_launch();
    }
    if (da) {
        adapter_grad_kernel<<<(unsigned)(((size_t)d->adapters * R * K + 255) / 256), 256, 0, s>>>(M, K, R, d->adapters, (const __nv_bfloat16*)x, ldx, u, nullptr, row_id, key, 1, da);
        count_launch();
    }
    if (db) {
        adapter_grad_kernel<<<(unsigned)(((size_t)d->adapters * R * N + 255) / 256), 256, 0, s>>>(M, N, R, d->adapters, (const __nv_bfloat16*)dy, lddy, t, scale, row_id, none, 0, db);
        count_launch();
    }
    return launch_status();
}
