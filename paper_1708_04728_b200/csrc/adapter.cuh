// What the kernels of the low-rank adapters share: which request a row belongs to, masks of neighbouring elements, launch parameters.
#pragma once
#include <cuda.h>

#include "common.cuh"
#include "dropout.cuh"

namespace dr {

constexpr int ROW_SHARED = -1;      // a row of a request without an adapter
constexpr int ROW_NONE = -2;        // a row of no request: left as it was

struct AdRows {
    int M, segments, adapters;
    const int *row_start, *adapter;
};

// Number of offsets row_start[lo .. hi) that are <= m, plus lo, by binary search.  Whatever the offsets hold, the search stays inside them.
__device__ __forceinline__ int offsets_upto(const AdRows& r, int m, int lo, int hi) {
    while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);
        if (__ldg(r.row_start + mid) <= m) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ int adapter_of_count(const AdRows& r, int count) {     // count: offsets <= the row
    if (count <= 0 || count > r.segments) return ROW_NONE;
    const int a = __ldg(r.adapter + count - 1);
    return a >= 0 && a < r.adapters ? a : ROW_SHARED;           // an adapter out of range is none
}
// The adapter of row m0 + lane, by a whole warp, with few dependent loads: up to 32 offsets are loaded at once and counted out of registers; of more, 32 are
// probed at a time (two loads for a thousand requests instead of ten) for the first and the last of the rows, and the ones between are counted.
__device__ __forceinline__ int offsets_counted(const AdRows& r, int m, int lo, int n, int lane) {     // n <= 32 offsets from lo on
    const int o = lane < n ? __ldg(r.row_start + lo + lane) : 0x7fffffff;
    int count = lo;
    for (int k = 0; k < n; ++k) count += __shfl_sync(0xffffffffu, o, k) <= m ? 1 : 0;
    return count;
}
__device__ __forceinline__ int adapter_of_warp_row(const AdRows& r, int m0, int lane) {
    const int m = m0 + lane;
    if (r.segments < 32) {
        const int count = offsets_counted(r, m, 0, r.segments + 1, lane);
        return m >= r.M ? ROW_NONE : adapter_of_count(r, count);
    }
    const int last = m0 + 31;
    int lo[2] = {0, 0}, n[2] = {r.segments + 1, r.segments + 1};
    while (n[0] > 0 || n[1] > 0) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (n[k] <= 0) continue;
            const int step = (n[k] + 31) >> 5;                  // lane probes the last offset of its piece
            const int at = min(lane * step + step - 1, n[k] - 1);
            const bool le = lane * step < n[k] && __ldg(r.row_start + lo[k] + at) <= (k ? last : m0);
            const unsigned below = __ballot_sync(0xffffffffu, le);
            const int pieces = __popc(below & ~(below + 1));    // the pieces in front of the first one that reaches beyond the row
            const int skip = min(pieces * step, n[k]);
            lo[k] += skip;
            n[k] = skip == n[k] ? 0 : min(step - 1, n[k] - skip - 1);   // the probed offset of the next piece is above the row
        }
    }
    const int between = lo[1] - lo[0];
    const int count = between <= 0 ? lo[0] : between <= 32 ? offsets_counted(r, m, lo[0], between, lane) : offsets_upto(r, m, lo[0], lo[1]);
    return m >= r.M ? ROW_NONE : adapter_of_count(r, count);
}

// ---- the adapters of a tile of rows, by 128 threads (barrier 1; bt their number) ---------------------------------------------
__device__ __forceinline__ void builders_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// the same, and whether any of them says so: they leave together or not at all, since this barrier has no limit
__device__ __forceinline__ bool builders_any(bool v) {
    uint32_t r;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbar.red.or.pred p, 1, 128, q;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(r) : "r"((uint32_t)v) : "memory");
    return r != 0;
}
struct ApFind {
    int lowest[4], highest[4];
    uint32_t bits[128];
    int before[128];
    int sums[4];
};
// The adapters in use among the rows whose adapters id[] are (N of them a thread): their list in ascending order, this thread's places in it (or id
// itself where that is none), and how many there are.
template <int N>
__device__ __forceinline__ int ap_find(ApFind& f, uint16_t* list, const int (&id)[N], int (&slot)[N], int bt) {
    const int lane = bt & 31, w = bt >> 5;
    int lo = 0x7fffffff, hi = -1;
#pragma unroll
    for (int h = 0; h < N; ++h) {
        lo = min(lo, id[h] >= 0 ? id[h] : 0x7fffffff);
        hi = max(hi, id[h]);
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    if (lane == 0) { f.lowest[w] = lo; f.highest[w] = hi; }
    f.bits[bt] = 0;
    builders_sync();
    lo = min(min(f.lowest[0], f.lowest[1]), min(f.lowest[2], f.lowest[3]));
    hi = max(max(f.highest[0], f.highest[1]), max(f.highest[2], f.highest[3]));
    if (hi < 0 || lo == hi) {                       // none, or one: most tiles
        if (bt == 0) list[0] = (uint16_t)max(hi, 0);
#pragma unroll
        for (int h = 0; h < N; ++h) slot[h] = id[h] >= 0 ? 0 : id[h];
        return hi < 0 ? 0 : 1;
    }
#pragma unroll
    for (int h = 0; h < N; ++h)
        if (id[h] >= 0) atomicOr(&f.bits[id[h] >> 5], 1u << (id[h] & 31));
    builders_sync();
    const uint32_t word = f.bits[bt];
    const int n = __popc(word);
    int incl = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    if (lane == 31) f.sums[w] = incl;
    builders_sync();
    int at = incl - n;
    for (int k = 0; k < w; ++k) at += f.sums[k];
    f.before[bt] = at;
    for (uint32_t x = word; x; x &= x - 1) list[at++] = (uint16_t)(bt * 32 + __ffs(x) - 1);
    builders_sync();
#pragma unroll
    for (int h = 0; h < N; ++h) slot[h] = id[h] >= 0 ? f.before[id[h] >> 5] + __popc(f.bits[id[h] >> 5] & ((1u << (id[h] & 31)) - 1u)) : id[h];
    return f.sums[0] + f.sums[1] + f.sums[2] + f.sums[3];
}

// The end of a CTA one of whose waits ran out, by all its threads: copies and MMAs in flight end within microseconds, then shared memory and TMEM may go.
__device__ __forceinline__ void ap_settle(volatile int* abort_flag) {
    __syncthreads();
    if (*abort_flag) {
        const long long t0 = clock64();
        while (clock64() - t0 < 400000ll) {}
        __syncthreads();
    }
}

// Which of 8 consecutive elements, the first with number e, are kept: bit i for element e + i.
__device__ __forceinline__ uint32_t drop_bits8(const DropKey& k, unsigned long long off, unsigned long long counter) {
    const uint4 w = drop_words(k, off, counter);
    uint32_t b = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) b |= drop_keep(w, i, k.thr) ? 1u << i : 0u;
    return b;
}
__device__ __forceinline__ uint32_t drop_bits8_at(const DropKey& k, unsigned long long off, unsigned long long e) {
    const int sh = (int)(e & 7);
    uint32_t b = 0;
#pragma unroll 1                                                 // one copy of the generator: the code has to stay in the instruction cache
    for (int i = 0; i < (sh ? 2 : 1); ++i) b |= drop_bits8(k, off, (e >> 3) + i) << (8 * i);
    return (b >> sh) & 0xFFu;
}
// 8 bfloat16 values, those whose bit is clear set to zero
__device__ __forceinline__ uint4 drop_apply8(uint4 v, uint32_t bits) {
    auto two = [](uint32_t u, uint32_t b) { return u & ((b & 1 ? 0xFFFFu : 0u) | (b & 2 ? 0xFFFF0000u : 0u)); };
    return make_uint4(two(v.x, bits), two(v.y, bits >> 2), two(v.z, bits >> 4), two(v.w, bits >> 6));
}

// Two float32 values as sums of three bfloat16 values each (all 24 bits; the first two of them alone 16 to 17), packed in pairs.
__device__ __forceinline__ void split3(float a, float b, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    hi = pack_bf16(a, b);
    // an infinity (or what rounds to one) has no remainder: inf - inf would be NaN
    const float ra = fabsf(bf16_lo(hi)) <= 3.4e38f ? a - bf16_lo(hi) : 0.f, rb = fabsf(bf16_hi(hi)) <= 3.4e38f ? b - bf16_hi(hi) : 0.f;
    mid = pack_bf16(ra, rb);
    lo = pack_bf16(ra - bf16_lo(mid), rb - bf16_hi(mid));
}

// A launch that may begin while the kernel in front of it ends (`overlap`): it then waits for that one before it reads what it wrote, in every CTA, so
// that what follows sees all of them complete.
template <class Kernel, class... Args>
static int start_kernel(Kernel k, const dim3& grid, int threads, int cluster_y, bool overlap, size_t smem, cudaStream_t s, const Args&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster_y > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = 1; attr[n].val.clusterDim.y = (unsigned)cluster_y; attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (overlap) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    if (cudaLaunchKernelEx(&cfg, k, args...) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
    count_launch();
    return DR_OK;
}

// ---- launches (adapter_down.cu, adapter_product.cu, adapter_grad.cu) -------------------------------------------------------
// t[m][r] = factor * sum_l D(z)[m][l] f_a[r][l], f [adapters * R][ldf] with 16-byte aligned rows and zeros behind L.  Written: in keep t itself, in rows
// of R (may be nullptr; zeros where a row has no adapter, nothing where it has no request); in out the bfloat16 terms of T = scale_a after t, [M][terms][Rp];
// in row_id each row's adapter
struct DownPlan { int mt, warps_k, rows_cta, ks, zsplit, rt, rchunks; bool tile; };
DownPlan adapter_down_plan(int M, int L, int R, int adapters, int segments, bool dropped);
int adapter_down_run(const DownPlan& plan, const AdRows& rows, int L, int R, int Rp, const __nv_bfloat16* z, size_t ldz, const __nv_bfloat16* f, size_t ldf,
                     const DropKey& key, float factor, const float* scale, float after, int terms, __nv_bfloat16* out, float* keep, int* row_id, bool overlap, cudaStream_t s);

// out[m][c] = act(sum_l z[m][l] w + bias[c] + D(T[m] f_a)):   forward w [C][ldw] (rows of l), f [adapters][C][R];
// transposed w [L][ldw] (rows of c), f [adapters][R][ldf]
struct ProductArgs {
    AdRows rows;
    int L, C, R, Rp;
    const __nv_bfloat16 *z, *w, *f;
    size_t ldz, ldw, ldf;
    const int* row_id;
    const __nv_bfloat16* t;     // [M][terms][Rp]; of the terms the result's type calls for are taken
    int terms;
    const float* bias;
    unsigned flags;
    void* out;
    size_t ldo;
    bool transposed;
    const uint32_t* mask;       // bits of what D keeps, rows of ldm words; nullptr: D is the identity (the forward pass')
    int ldm;
};
int adapter_product_run(const ProductArgs& a, bool overlap, cudaStream_t s);

// g_a[r][c] = sum over the rows of adapter a of P[m][r] D(z)[m][c]
struct GradJob {
    int C;
    const __nv_bfloat16* z;
    size_t ldz;
    const __nv_bfloat16* p;     // P as three bfloat16 values, [M][3][Rp]
    const uint32_t* mask;       // as in ProductArgs
    int ldm;
    float* out;                 // [adapters][R][C], or [adapters][C][R] where swap
    int swap;
};
struct GradPlan { int tiles, splits, rn, rchunks; size_t perm, start, terms, part[2], bytes; };
GradPlan adapter_grad_plan(int M, int R, int adapters, const int C[2]);
int adapter_grad_run(const GradPlan& plan, const AdRows& rows, int R, const GradJob jobs[2], char* ws, bool overlap, cudaStream_t s);
// in one launch, each where its result is wanted: the rows sorted by adapter (perm, start), b [adapters][N][R] turned to bt [adapters][R][ldb] with zeros
// behind N, scale_a t as three bfloat16 values, the dropout's mask over [M][K] (a bit each: drawn once, and read by both products that want it)
int adapter_prep_run(const AdRows& rows, int* perm, int* start, int N, int R, int Rp, const __nv_bfloat16* b, __nv_bfloat16* bt, size_t ldb, const float* t,
                     const float* scale, __nv_bfloat16* terms, const DropKey& key, int K, uint32_t* mask, int ldm, cudaStream_t s);

// rows of `cols` elements, `ld` apart, as rows of ldd >= cols (a multiple of 8) with zeros behind them; at most four tensors
struct AlignJob { const __nv_bfloat16* src; size_t ld; __nv_bfloat16* dst; size_t ldd, rows; int cols; };
int adapter_align_run(const AlignJob* jobs, int n, cudaStream_t s);
}  // namespace dr
