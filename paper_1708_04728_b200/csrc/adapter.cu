// A 1 x 1 (or fully connected) layer with the low-rank adapters of many requests beside its shared filters, forward and backward:
//   t = D(x) A_a^T,  y = act(x W^T + bias + scale_a t B_a^T);     u = scale_a dy B_a,  dx = dy W + D(u A_a),  dA_a = sum u^T D(x),
//   dB_a = scale_a sum dy^T t,     a the adapter of the request that a row belongs to, D the dropout of dropout.cuh.
// Arguments, workspaces and the order of the kernels: adapter_down.cu (t and u), adapter_product.cu (y and dx), adapter_grad.cu (dA and dB).
#include "adapter.cuh"

namespace dr {

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

// Places in the workspace.  Rows that are not on 16-byte boundaries are laid out there first: 16-byte loads and TMA want them so.
struct Places {
    size_t bytes = 0;
    size_t take(size_t n) { const size_t at = bytes; bytes += up256(n); return at; }
};
static int up8(int n) { return (n + 7) & ~7; }

struct ForwardPlan {
    DownPlan down;
    int Kp, Rp, terms;
    bool copy_x, copy_k;        // x; w and a
    size_t ids, t, x, w, a, bytes;
};
static ForwardPlan forward_plan(const dr_adapter_desc* d, int M, int ldx, int segments) {
    ForwardPlan f;
    f.down = adapter_down_plan(M, d->Cin, d->rank, d->adapters, segments, d->drop_p > 0.f);
    f.Kp = up8(d->Cin);
    f.Rp = up8(d->rank);
    f.copy_k = d->Cin & 7;
    f.copy_x = f.copy_k || (ldx & 7);
    Places at;
    f.ids = at.take((size_t)M * 4);
    f.terms = (d->flags & DR_OUT_F32) ? 3 : 2;
    f.t = at.take((size_t)M * f.terms * f.Rp * 2);
    f.x = at.take(f.copy_x ? (size_t)M * f.Kp * 2 : 0);
    f.w = at.take(f.copy_k ? (size_t)d->Cout * f.Kp * 2 : 0);
    f.a = at.take(f.copy_k ? (size_t)d->adapters * d->rank * f.Kp * 2 : 0);
    f.bytes = at.bytes;
    return f;
}

struct BackwardPlan {
    DownPlan down;
    GradPlan grad;
    int Kp, Np, Rp;
    bool copy_x, copy_k, copy_dy;
    int ldm;                    // words of a row of the mask: whole 64 channels
    size_t ids, u, x, w, a, dy, bt, mask, g, bytes;
};
static BackwardPlan backward_plan(const dr_adapter_desc* d, int M, int ldx, int lddy, int segments) {
    BackwardPlan f;
    f.down = adapter_down_plan(M, d->Cout, d->rank, d->adapters, segments, false);
    const int C[2] = {d->Cin, d->Cout};
    f.grad = adapter_grad_plan(M, d->rank, d->adapters, C);
    f.Kp = up8(d->Cin);
    f.Np = up8(d->Cout);
    f.Rp = up8(d->rank);
    f.copy_k = d->Cin & 7;
    f.copy_x = f.copy_k || (ldx & 7);
    f.copy_dy = (d->Cout & 7) || (lddy & 7);
    Places at;
    f.ids = at.take((size_t)M * 4);
    f.u = at.take((size_t)M * 3 * f.Rp * 2);
    f.x = at.take(f.copy_x ? (size_t)M * f.Kp * 2 : 0);
    f.w = at.take(f.copy_k ? (size_t)d->Cout * f.Kp * 2 : 0);
    f.a = at.take(f.copy_k ? (size_t)d->adapters * d->rank * f.Kp * 2 : 0);
    f.dy = at.take(f.copy_dy ? (size_t)M * f.Np * 2 : 0);
    f.bt = at.take((size_t)d->adapters * d->rank * f.Np * 2);
    f.ldm = (d->Cin + 63) / 64 * 2;
    f.mask = at.take(d->drop_p > 0.f ? (size_t)M * f.ldm * 4 : 0);
    f.g = at.take(f.grad.bytes);
    f.bytes = at.bytes;
    return f;
}
// The tensors themselves, or their aligned copies, all made in one launch.
struct Aligner {
    AlignJob job[4];
    int n = 0;
    char* ws;
    explicit Aligner(char* workspace) : ws(workspace) {}
    void place(bool copy, size_t rows, int cols, int colsp, const void* src, size_t ld, size_t at, const __nv_bfloat16** p, size_t* ldp) {
        *p = copy ? (const __nv_bfloat16*)(ws + at) : (const __nv_bfloat16*)src;
        *ldp = copy ? (size_t)colsp : ld;
        if (copy) job[n++] = {(const __nv_bfloat16*)src, ld, (__nv_bfloat16*)(ws + at), (size_t)colsp, rows, cols};
    }
};

}  // namespace dr

using namespace dr;

extern "C" int dr_adapter_workspace_bytes(const dr_adapter_desc* d, int M, int ldx, size_t* bytes) {
    const int rc = desc_check(d, M);
    if (rc != DR_OK) return rc;
    if (!bytes || ld_check(&ldx, d->Cin) != DR_OK) return DR_ERR_INVALID_ARG;
    *bytes = forward_plan(d, M, ldx, 1).bytes;
    return DR_OK;
}

extern "C" int dr_adapter_bwd_workspace_bytes(const dr_adapter_desc* d, int M, int ldx, int lddy, size_t* bytes) {
    const int rc = desc_check(d, M);
    if (rc != DR_OK) return rc;
    if (!bytes || ld_check(&ldx, d->Cin) != DR_OK || ld_check(&lddy, d->Cout) != DR_OK) return DR_ERR_INVALID_ARG;
    *bytes = backward_plan(d, M, ldx, lddy, 1).bytes;
    return DR_OK;
}

extern "C" int dr_adapter(const dr_adapter_desc* d, int M, const void* x, int ldx, const void* w, const float* bias, const void* a, const void* b,
                          const float* scale, int segments, const int* row_start, const int* adapter, void* y, int ldy, float* t,
                          const unsigned long long* step, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = desc_check(d, M);
    if (rc != DR_OK) return rc;
    if (ld_check(&ldx, d->Cin) != DR_OK || ld_check(&ldy, d->Cout) != DR_OK || segments < 0) return DR_ERR_INVALID_ARG;
    if (segments > DR_ADAPTER_MAX_ROWS) return DR_ERR_UNSUPPORTED;
    if (M == 0 || segments == 0) return DR_OK;
    if (!x || !w || !a || !b || !y || !row_start || !adapter || !workspace || ((d->flags & DR_BIAS) && !bias)) return DR_ERR_INVALID_ARG;
    if (!aligned16(x) || !aligned16(w) || !aligned16(a) || !aligned16(b) || ((uintptr_t)y & ((d->flags & DR_OUT_F32) ? 3 : 1)) || ((uintptr_t)bias & 3) ||
        ((uintptr_t)scale & 3) || ((uintptr_t)row_start & 3) || ((uintptr_t)adapter & 3) || ((uintptr_t)t & 3) || ((uintptr_t)step & 7) ||
        ((uintptr_t)workspace & 255))
        return DR_ERR_ALIGNMENT;
    const ForwardPlan f = forward_plan(d, M, ldx, segments);
    if (workspace_bytes < f.bytes) return DR_ERR_WORKSPACE;
    const cudaStream_t s = (cudaStream_t)stream;
    char* const ws = (char*)workspace;
    const int K = d->Cin, N = d->Cout, R = d->rank;
    const AdRows rows = {M, segments, d->adapters, row_start, adapter};
    const DropKey key = drop_key(d->drop_p, d->drop_seed, d->drop_offset, step);
    const __nv_bfloat16 *xp, *wp, *ap;
    size_t ldxp, ldwp, ldap;
    Aligner al(ws);
    al.place(f.copy_x, M, K, f.Kp, x, ldx, f.x, &xp, &ldxp);
    al.place(f.copy_k, N, K, f.Kp, w, K, f.w, &wp, &ldwp);
    al.place(f.copy_k, (size_t)d->adapters * R, K, f.Kp, a, K, f.a, &ap, &ldap);
    if ((rc = adapter_align_run(al.job, al.n, s)) != DR_OK) return rc;
    __nv_bfloat16* const tw = (__nv_bfloat16*)(ws + f.t);
    int* const ids = (int*)(ws + f.ids);
    rc = adapter_down_run(f.down, rows, K, R, f.Rp, xp, ldxp, ap, ldap, key, key.thr ? key.scale : 1.f, scale, 1.f, f.terms, tw, t, ids, false, s);
    if (rc != DR_OK) return rc;
    const ProductArgs g = {rows, K, N, R, f.Rp, xp, wp, (const __nv_bfloat16*)b, ldxp, ldwp, 0, ids, tw, f.terms, bias, d->flags, y, (size_t)ldy, false, nullptr, 0};
    return adapter_product_run(g, true, s);
}

extern "C" int dr_adapter_bwd(const dr_adapter_desc* d, int M, const void* dy, int lddy, const void* x, int ldx, const void* w, const void* a, const void* b,
                              const float* scale, int segments, const int* row_start, const int* adapter, const float* t, void* dx, int lddx, float* da,
                              float* db, const unsigned long long* step, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = desc_check(d, M);
    if (rc != DR_OK) return rc;
    if (ld_check(&ldx, d->Cin) != DR_OK || ld_check(&lddx, d->Cin) != DR_OK || ld_check(&lddy, d->Cout) != DR_OK || segments < 0) return DR_ERR_INVALID_ARG;
    if (segments > DR_ADAPTER_MAX_ROWS) return DR_ERR_UNSUPPORTED;              // numbers of requests are counted in 32 bits, 256 ahead
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
    const BackwardPlan f = backward_plan(d, M, ldx, lddy, segments);
    if (workspace_bytes < f.bytes) return DR_ERR_WORKSPACE;
    if (!dx && !da && !db) return DR_OK;
    char* const ws = (char*)workspace;
    const AdRows rows = {M, segments, d->adapters, row_start, adapter};
    const DropKey key = drop_key(d->drop_p, d->drop_seed, d->drop_offset, step), none = drop_key(0., 0, 0, nullptr);
    const float kept = key.thr ? key.scale : 1.f;
    const __nv_bfloat16 *dyp, *xp = nullptr, *wp = nullptr, *ap = nullptr;
    size_t lddyp, ldxp = 0, ldwp = 0, ldap = 0;
    Aligner al(ws);
    al.place(f.copy_dy, M, N, f.Np, dy, lddy, f.dy, &dyp, &lddyp);
    if (da) al.place(f.copy_x, M, K, f.Kp, x, ldx, f.x, &xp, &ldxp);
    if (dx) al.place(f.copy_k, N, K, f.Kp, w, K, f.w, &wp, &ldwp);
    if (dx) al.place(f.copy_k, (size_t)d->adapters * R, K, f.Kp, a, K, f.a, &ap, &ldap);
    if ((rc = adapter_align_run(al.job, al.n, s)) != DR_OK) return rc;
    __nv_bfloat16* const u = (__nv_bfloat16*)(ws + f.u);
    int* const ids = (int*)(ws + f.ids);
    const bool grads = da || db, u_wanted = dx || da;
    __nv_bfloat16* const bt = (__nv_bfloat16*)(ws + f.bt);
    __nv_bfloat16* const terms = (__nv_bfloat16*)(ws + f.g + f.grad.terms);
    uint32_t* const mask = key.thr && u_wanted ? (uint32_t*)(ws + f.mask) : nullptr;
    rc = adapter_prep_run(rows, grads ? (int*)(ws + f.g + f.grad.perm) : nullptr, (int*)(ws + f.g + f.grad.start), N, R, f.Rp, (const __nv_bfloat16*)b,
                          u_wanted ? bt : nullptr, f.Np, t, scale, db ? terms : nullptr, key, K, mask, f.ldm, s);
    if (rc != DR_OK) return rc;
    // The lists are made by one block for each adapter, 4 ns for each request of the call: where they are many the first product begins once that is done, and
    // with it the second, whose waits have a limit of two seconds.
    const bool overlap = segments <= 1 << 22;
    if (u_wanted && (rc = adapter_down_run(f.down, rows, N, R, f.Rp, dyp, lddyp, bt, f.Np, none, 1.f, scale, kept, 3, u, nullptr, ids, overlap, s)) != DR_OK) return rc;
    if (dx) {
        const ProductArgs g = {rows, N, K, R, f.Rp, dyp, wp, ap, lddyp, ldwp, ldap, ids, u, 3, nullptr, 0, dx, (size_t)lddx, true, mask, f.ldm};
        if ((rc = adapter_product_run(g, true, s)) != DR_OK) return rc;
    }
    if (da || db) {
        const GradJob jobs[2] = {{K, xp, ldxp, u, mask, f.ldm, da, 0}, {N, dyp, lddyp, terms, nullptr, 0, db, 1}};
        if ((rc = adapter_grad_run(f.grad, rows, R, jobs, ws + f.g, true, s)) != DR_OK) return rc;
    }
    return DR_OK;
}
