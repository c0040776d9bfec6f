// The adapters' gradients, g_a[r][c] = sum over the rows m of adapter a of P[m][r] D(z)[m][c]: with P = u and z = x the first factor's,
// with P = t and z = dy the second's.  Bound by the bytes of z.
//
// The rows are sorted by adapter first (an index list; order within an adapter as in the tensor).  A CTA owns a column block and an even share of the
// sorted rows, whatever their adapters; where its share passes from one adapter to the next it writes what it has and starts over.  Share
// and adapter only grow along the list, so their sum numbers the partial results without gaps; they are added in order by a second
// kernel: the same result on every run, and no share is larger than another however the requests are spread.
//
// Warps multiply fragments (mma.sync) of P^T (rows: r) and z (columns: c).  A thread loads 8 neighbouring columns of four rows: with
// the columns of eight tiles interleaved (column 8 g + n is column g of tile n) and four neighbouring rows to a thread its loads are 16 bytes wide
// and the transposition is a byte permutation in registers.  P enters as the sum of two bfloat16 values.
#include <algorithm>

#include "adapter.cuh"

namespace dr {

// perm: rows sorted by adapter; start[a]: where adapter a's begin, start[adapters]: how many there are.  A block per adapter.
__global__ void __launch_bounds__(256) adapter_sort_kernel(const AdRows r, int* __restrict__ perm, int* __restrict__ start) {
    __shared__ int sum_own[8], sum_less[8];
    const int a = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto length = [&](int s, int& id, int& first) {
        if (s >= r.segments) { id = ROW_NONE; first = 0; return 0; }
        first = min(max(__ldg(r.row_start + s), 0), r.M);
        const int last = min(max(__ldg(r.row_start + s + 1), first), r.M);
        id = __ldg(r.adapter + s);
        if (id < 0 || id >= r.adapters) id = ROW_SHARED;
        return last - first;
    };
    // how many rows belong to adapters in front of this one, and to this one
    long long less = 0, own = 0;
    for (int s = threadIdx.x; s < r.segments; s += 256) {
        int id, first;
        const int n = length(s, id, first);
        if (id >= 0 && id < a) less += n;
        if (id == a) own += n;
    }
    for (int o = 16; o; o >>= 1) { less += __shfl_xor_sync(0xffffffffu, less, o); own += __shfl_xor_sync(0xffffffffu, own, o); }
    if (lane == 0) { sum_less[warp] = (int)min(less, (long long)r.M); sum_own[warp] = (int)min(own, (long long)r.M); }
    __syncthreads();
    long long base = 0, count = 0;
    for (int w = 0; w < 8; ++w) { base += sum_less[w]; count += sum_own[w]; }
    // offsets that decrease may count rows twice: the list ends at M
    base = min(base, (long long)r.M);
    if (threadIdx.x == 0) {
        start[a] = (int)base;
        if (a == r.adapters - 1) start[r.adapters] = (int)min(base + count, (long long)r.M);
    }
    if (count == 0) return;
    for (int s0 = 0; s0 < r.segments; s0 += 256) {
        int id, first;
        int n = length(s0 + (int)threadIdx.x, id, first);
        if (id != a) n = 0;
        int incl = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        __syncthreads();
        if (lane == 31) sum_own[warp] = incl;
        __syncthreads();
        int at = incl - n, total = 0;
        for (int w = 0; w < 8; ++w) { if (w < warp) at += sum_own[w]; total += sum_own[w]; }
        // a warp writes the rows of its own segments one after the other
        for (unsigned some = __ballot_sync(0xffffffffu, n > 0); some; some &= some - 1) {
            const int k = __ffs(some) - 1;
            const int len = __shfl_sync(0xffffffffu, n, k), f = __shfl_sync(0xffffffffu, first, k);
            const long long to = base + __shfl_sync(0xffffffffu, at, k);
            for (int i = lane; i < len; i += 32)
                if (to + i < r.M) perm[to + i] = f + i;
        }
        base += total;
    }
}

struct GradParams {
    int M, R, adapters, splits, rchunks;
    const int *perm, *start;
    int blocks0;                // column blocks of the first job
    struct Job {
        int C, ldp, swap;
        const __nv_bfloat16* z;
        size_t ldz;
        const float *p, *scale;
        const __nv_bfloat16* terms;
        DropKey key;
        float *part, *out;
    } job[2];
};

__device__ __forceinline__ void mma_bf16_g(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A CTA: 64 columns, RT tiles of 16 r; its 8 warps take every eighth 16 rows.
template <int RT>
__global__ void __launch_bounds__(256) adapter_grad_kernel(const GradParams p) {
    extern __shared__ float gr_join[];                           // [8 warps][RT * 16][65], half of them at a time
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int which = (int)blockIdx.x >= p.blocks0;
    const GradParams::Job& j = p.job[which];
    const int cb = (int)blockIdx.x - (which ? p.blocks0 : 0);
    const int split = blockIdx.y, r0 = (int)blockIdx.z * RT * 16;
    const int total = min(max(__ldg(p.start + p.adapters), 0), p.M);
    const int share = ((total + p.splits - 1) / p.splits + 15) & ~15;
    const int from = min(split * share, total), to = min(from + share, total);
    if (from >= to) return;
    const int c = cb * 64 + 8 * g;
    const unsigned long long off = j.key.thr ? drop_offset(j.key) : 0ull;
    const bool whole = (j.C & 7) == 0;
    // first adapter of the share: the last one that begins at or in front of it and is not empty
    int lo = 0, hi = p.adapters;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(p.start + mid + 1) <= from) lo = mid + 1;
        else hi = mid;
    }
    for (int a = lo; a < p.adapters; ++a) {
        const int u = max(from, __ldg(p.start + a)), v = min(to, __ldg(p.start + a + 1));
        if (__ldg(p.start + a) >= to) break;
        if (u >= v) continue;
        const float w = j.scale ? __ldg(j.scale + a) : 1.f;
        float acc[RT][8][4] = {};
        for (int i = u + 16 * warp; i < v; i += 128) {
            uint4 z[4];
            int row[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = i + 4 * q + k;
                row[k] = at < v ? (int)min((unsigned)__ldg(p.perm + at), (unsigned)(p.M - 1)) : -1;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                z[k] = make_uint4(0, 0, 0, 0);
                if (row[k] >= 0 && c < j.C) z[k] = __ldg(reinterpret_cast<const uint4*>(j.z + (size_t)row[k] * j.ldz + c));
            }
            uint32_t ph[RT][4], pm[RT][4], pl[RT][4];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                float x[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int r = r0 + 16 * t + 8 * h + g;
                        float s = 0.f;
                        if (row[k] >= 0 && r < p.R)
{
                            if (j.terms) {
                                const __nv_bfloat16* u = j.terms + (size_t)row[k] * 3 * j.ldp + r;
                                s = (__bfloat162float(u[0]) + __bfloat162float(u[j.ldp])) + __bfloat162float(u[2 * j.ldp]);
                            } else {
                                s = __ldg(j.p + (size_t)row[k] * j.ldp + r) * w;
                            }
                        }
                        x[h][k] = s;
                    }
                split3(x[0][0], x[0][1], ph[t][0], pm[t][0], pl[t][0]);
                split3(x[1][0], x[1][1], ph[t][1], pm[t][1], pl[t][1]);
                split3(x[0][2], x[0][3], ph[t][2], pm[t][2], pl[t][2]);
                split3(x[1][2], x[1][3], ph[t][3], pm[t][3], pl[t][3]);
            }
            if (j.key.thr) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const unsigned long long e = (unsigned long long)max(row[k], 0) * j.C + c;
                    z[k] = drop_apply8(z[k], whole ? drop_bits8(j.key, off, e >> 3) : drop_bits8_at(j.key, off, e));
                }
            }
            const uint32_t* zu = reinterpret_cast<const uint32_t*>(z);
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                const uint32_t sel = (n & 1) ? 0x7632u : 0x5410u;
                const uint32_t b0 = __byte_perm(zu[n >> 1], zu[4 + (n >> 1)], sel), b1 = __byte_perm(zu[8 + (n >> 1)], zu[12 + (n >> 1)], sel);
#pragma unroll
                for (int t = 0; t < RT; ++t) {
                    mma_bf16_g(acc[t][n], ph[t], b0, b1);
                    mma_bf16_g(acc[t][n], pm[t], b0, b1);
                    mma_bf16_g(acc[t][n], pl[t], b0, b1);
                }
            }
        }
        // the warps' sums, in order: column 8 * (2 q + i) + n of tile n's column 2 q + i
        float* mine = gr_join + (size_t)warp * (RT * 16) * 65;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) mine[(16 * t + 8 * (i >> 1) + g) * 65 + 8 * (2 * q + (i & 1)) + n] = acc[t][n][i];
        __syncthreads();
        float* part = j.part + (size_t)(split + a) * p.R * j.C;
        for (int i = threadIdx.x; i < RT * 16 * 64; i += 256) {
            const int r = i >> 6, cc = i & 63;
            if (r0 + r >= p.R || cb * 64 + cc >= j.C) continue;
            float s = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) s += gr_join[((size_t)k * (RT * 16) + r) * 65 + cc];
            part[(size_t)(r0 + r) * j.C + cb * 64 + cc] = s;
        }
    }
}

__global__ void __launch_bounds__(256) adapter_grad_join_kernel(const GradParams p, int from_job) {
    const int which = from_job + (int)blockIdx.z;
    const GradParams::Job& j = p.job[which];
    if (!j.out) return;
    const int a = blockIdx.y;
    const int total = min(max(__ldg(p.start + p.adapters), 0), p.M);
    const int share = ((total + p.splits - 1) / p.splits + 15) & ~15;
    const int u = __ldg(p.start + a), v = min(__ldg(p.start + a + 1), total);
    const int n = p.R * j.C;
    const int s0 = u < v ? u / share : 0, s1 = u < v ? (v - 1) / share : -1;
    for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
        float s = 0.f;
        for (int k = s0; k <= s1; ++k) s += j.part[(size_t)(k + a) * n + i];
        const int r = i / j.C, c = i - r * j.C;
        j.out[(size_t)a * n + (j.swap ? (size_t)c * p.R + r : (size_t)i)] = s;
    }
}

GradPlan adapter_grad_plan(int M, int R, int adapters, const int C[2]) {
    GradPlan g = {};
    g.rt = R <= 16 ? 1 : R <= 32 ? 2 : 4;
    g.rchunks = (R + 16 * g.rt - 1) / (16 * g.rt);
    const int blocks = ((C[0] + 63) / 64 + (C[1] + 63) / 64) * g.rchunks;
    g.splits = std::max(1, std::min((M + 127) / 128, (4 * num_sms() + blocks - 1) / blocks));
    size_t at = 0;
    auto take = [&](size_t& where, size_t bytes) { where = at; at += (bytes + 255) / 256 * 256; };
    take(g.perm, (size_t)M * 4);
    take(g.start, (size_t)(adapters + 1) * 4);
    for (int k = 0; k < 2; ++k) take(g.part[k], (size_t)(g.splits + adapters - 1) * R * C[k] * 4);
    g.bytes = at;
    return g;
}

int adapter_sort_run(const AdRows& rows, int* perm, int* start, cudaStream_t s) {
    adapter_sort_kernel<<<(unsigned)rows.adapters, 256, 0, s>>>(rows, perm, start);
    count_launch();
    return launch_status();
}

template <int RT>
static int grad_launch(const dim3& grid, const GradParams& p, cudaStream_t s) {
    constexpr int smem = 8 * RT * 16 * 65 * 4;
    static PerDeviceFlag ready;
    if (!ready.get()) {
        if (cudaFuncSetAttribute(adapter_grad_kernel<RT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
        ready.set();
    }
    adapter_grad_kernel<RT><<<grid, 256, smem, s>>>(p);
    return launch_status();
}

int adapter_grad_run(const GradPlan& plan, const AdRows& rows, int R, const GradJob jobs[2], char* ws, cudaStream_t s) {
    GradParams p = {};
    p.M = rows.M; p.R = R; p.adapters = rows.adapters; p.splits = plan.splits; p.rchunks = plan.rchunks;
    p.perm = (int*)(ws + plan.perm); p.start = (int*)(ws + plan.start);
    int blocks[2], most = 0;
    for (int k = 0; k < 2; ++k) {
        const GradJob& g = jobs[k];
        p.job[k] = {g.C, g.ldp, g.swap, g.z, g.ldz, g.p, g.scale, g.terms, g.key, (float*)(ws + plan.part[k]), g.out};
        blocks[k] = g.out ? (g.C + 63) / 64 : 0;
        if (g.out) most = std::max(most, g.C);
    }
    p.blocks0 = blocks[0];
    const dim3 grid((unsigned)(blocks[0] + blocks[1]), (unsigned)plan.splits, (unsigned)plan.rchunks);
    const int rc = plan.rt == 1 ? grad_launch<1>(grid, p, s) : plan.rt == 2 ? grad_launch<2>(grid, p, s) : grad_launch<4>(grid, p, s);
    if (rc != DR_OK) return rc;
    const long long n = ((long long)R * most + 255) / 256;
    adapter_grad_join_kernel<<<dim3((unsigned)std::min(n, 1024ll), (unsigned)rows.adapters, 2), 256, 0, s>>>(p, 0);
    count_launch(2);
    return launch_status();
}

}  // namespace dr
