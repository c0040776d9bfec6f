// The orthogonalised update of matrices with at most 128 rows (after transposing a tall one), a thread-block cluster per matrix.
//
// What bounds such a matrix is not its arithmetic but 15 dependent products, so nothing leaves the SM that does not have to.  A CTA
// keeps a slab of X's columns in shared memory for all steps, as float16 pairs in the layout that serves both as rows of X (A = X X^T,
// contraction along the slab) and as the second operand of F X.  Per step
//   A    each CTA multiplies its slab by its own transpose; the parts are summed through global memory, every CTA the columns it
//        owns, and E (A without its diagonal) and the diagonal go to all CTAs' shared memory: two cluster barriers,
//   F    every CTA computes E E and the polynomial for itself: one 128 x 128 product is cheaper than another exchange,
//   X    every CTA updates its slab in place.
// Products and element-wise terms as in the kernel for larger matrices (muon.cu); with few rows rounding errors average less, so
// matrices of up to 64 rows multiply hi hi + hi lo + lo hi: the tensor cores idle here either way.
#include <algorithm>
#include <cmath>
#include <mutex>

#include "muon_common.cuh"

namespace dr {

constexpr int NSS_THREADS = 256;
constexpr int NSS_CHUNK = 128 * 128;        // 64 columns of 128 rows
constexpr int NSS_MAX_CHUNKS = 4;           // of a CTA's slab: 64 KB hi, 64 KB lo
// Always asked for in full: one CTA per SM.  A second one there would wait for the first one's tensor memory, and the first, at a
// cluster barrier, for the second.
constexpr int NSS_SMEM = 2 * NSS_MAX_CHUNKS * NSS_CHUNK + 4 * NSS_CHUNK + 1024;
static_assert(NSS_SMEM > 114 * 1024, "two CTAs must not fit an SM");

struct NsSmall {
    NsInput in;
    int batch, steps, n, m, G, groups, chunks, terms;
    float coef[3 * DR_NS_MAX_STEPS];
    float* part;                // [group][CTA][column][128 rows]: parts of A
    int* status;
};

struct NsSmallShared {
    uint64_t done;
    uint32_t tmem_base;
    int abort;
    double red[8], norm[16];
    float d[128], rs[128];
};

// byte offset of 8 columns (one 16-byte unit) of a row inside [chunk][128 rows][128 bytes], 128-byte swizzle
__device__ __forceinline__ uint32_t nss_at(int row, int unit) { return (unit >> 3) * NSS_CHUNK + row * 128 + (((unit & 7) ^ (row & 7)) << 4); }
__device__ __forceinline__ void nss_ld(const uint8_t* base, int row, int unit, uint32_t* u) {
    const uint4 v = *reinterpret_cast<const uint4*>(base + nss_at(row, unit));
    u[0] = v.x; u[1] = v.y; u[2] = v.z; u[3] = v.w;
}
__device__ __forceinline__ void nss_st(uint8_t* base, int row, int unit, const uint32_t* u) {
    *reinterpret_cast<uint4*>(base + nss_at(row, unit)) = make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ void nss_st_remote(uint32_t addr, int cta, const uint32_t* u) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(mapa_shared(addr, cta)), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]) : "memory");
}

// 8 values of U at (row i, columns c .. c + 7) of X (zero past m); `at` is the first one's place in the user's matrix
__device__ __forceinline__ void nss_value(const NsSmall& p, size_t base, int i, int c, float* u) {
    const NsInput& in = p.in;
    if (!in.tall && in.vec && c < p.m) {
        ns_value<8>(in, base + (size_t)i * in.cols + c, u);
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        u[k] = 0.f;
        if (c + k < p.m) ns_value<1>(in, base + (in.tall ? (size_t)(c + k) * in.cols + i : (size_t)i * in.cols + c + k), u + k);
    }
}
__device__ __forceinline__ double nss_momentum(const NsSmall& p, size_t base, int i, int c) {
    const NsInput& in = p.in;
    if (!in.tall && in.vec && c < p.m) return ns_momentum_part<8>(in, base + (size_t)i * in.cols + c, 1, 0, 1);
    double s = 0.;
    for (int k = 0; k < 8; ++k)
        if (c + k < p.m) s += ns_momentum_part<1>(in, base + (in.tall ? (size_t)(c + k) * in.cols + i : (size_t)i * in.cols + c + k), 1, 0, 1);
    return s;
}

__global__ void __launch_bounds__(NSS_THREADS, 1) ns_small_kernel(const __grid_constant__ NsSmall p) {
    extern __shared__ uint8_t nss_raw[];
    __shared__ NsSmallShared sh;
    const uint32_t smem = (smem_u32(nss_raw) + 1023u) & ~1023u;
    uint8_t* const X = nss_raw + (smem - smem_u32(nss_raw));           // hi chunks, then lo chunks
    const int xlo = p.chunks * NSS_CHUNK, e_at = 2 * xlo;
    const int kc = (p.n + 63) / 64, elo = kc * NSS_CHUNK;              // chunks of an n x n operand
    uint8_t* const E = X + e_at;                                       // E, later F: hi, then lo
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int q = warp & 3, half = warp >> 2, row = q * 32 + lane;
    const int group = blockIdx.x / p.G, rank = blockIdx.x - group * p.G;
    const int c0 = rank * p.chunks * 64, units = p.chunks * 8;         // the slab: first column, 8-column units
    volatile int* abort_flag = &sh.abort;
    if (threadIdx.x == 0) {
        mbar_init(&sh.done, 1);
        sh.abort = 0;
        fence_barrier_init();
    }
    if (warp == 0) { tmem_alloc(&sh.tmem_base, 512); tmem_relinquish(); }
    // rows past n and columns past m or n take part in the products: zero, and never written again
    for (int i = threadIdx.x; i < (2 * p.chunks + 2 * kc) * (NSS_CHUNK / 16); i += NSS_THREADS) reinterpret_cast<uint4*>(X)[i] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x < 128) sh.d[threadIdx.x] = sh.rs[threadIdx.x] = 0.f;
    tc_fence_before();
    __syncthreads();
    if (p.G > 1) cluster_sync_all();            // every CTA runs before another writes to its shared memory
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base, acc_a = tmem, acc_x = tmem + 256;
    uint32_t phase = 0;

    // products: operands written by these threads through the other proxy; every thread returns when the product is done
    auto run = [&](auto issue) {
        fence_proxy_async_smem();
        tc_fence_before();
        __syncthreads();
        if (warp == 0 && elect_one()) {
            tc_fence_after();
            issue();
            umma_commit(&sh.done);
        }
        __syncwarp();
        if (!__all_sync(0xffffffffu, mbar_wait(&sh.done, phase, abort_flag))) {
            if (lane == 0 && !*abort_flag) report_timeout(p.status, 76, group);
            *abort_flag = 1;
        }
        phase ^= 1;
        tc_fence_after();
    };
    auto meet = [&]() {
        if (p.G > 1) cluster_sync_all();
        else __syncthreads();
    };
    // D += P Q^T over `kchunks` chunks of 64, both operands with the contraction along their rows
    auto product = [&](uint32_t d, uint32_t pa, uint32_t qa, int kchunks, int N, uint32_t accumulate) {
        const uint32_t idesc = (1u << 4) | ((uint32_t)(N >> 3) << 17) | (8u << 24);
        for (int k = 0; k < kchunks; ++k, pa += NSS_CHUNK, qa += NSS_CHUNK)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                umma_bf16_lo<false>(d, sdesc_lo(pa) + 2 * s, sdesc_lo(qa) + 2 * s, idesc, accumulate, 1u);
                accumulate = 1;
            }
    };

    for (int b = group; b < p.batch; b += p.groups) {
        const size_t base = (size_t)b * p.n * p.m;
        // v, and the sum of the squares of U: tall matrices are read along their rows, which are X's columns
        double s = 0.;
        for (int u = threadIdx.x; u < p.n * units; u += NSS_THREADS) {
            const int i = p.in.tall ? u % p.n : u / units, c = (p.in.tall ? u / p.n : u % units) * 8 + c0;
            if (c < p.m) s += nss_momentum(p, base, i, c);
        }
        s = ns_warp_sum(s);
        if (lane == 0) sh.red[warp] = s;
        __syncthreads();
        if (threadIdx.x < p.G) {
            s = 0.;
            for (int i = 0; i < NSS_THREADS / 32; ++i) s += sh.red[i];
            if (p.G > 1) asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(mapa_shared(smem_u32(&sh.norm[rank]), threadIdx.x)), "d"(s) : "memory");
            else sh.norm[0] = s;
        }
        meet();
        s = 0.;
        for (int i = 0; i < p.G; ++i) s += sh.norm[i];
        const float inv = (float)((double)NS_SCALE / (sqrt(s) + (double)p.in.eps));
        for (int u = threadIdx.x; u < p.n * units; u += NSS_THREADS) {
            const int i = p.in.tall ? u % p.n : u / units, w = p.in.tall ? u / p.n : u % units;
            alignas(8) float f[8];
            uint32_t h[4], l[4];
            nss_value(p, base, i, c0 + w * 8, f);
#pragma unroll
            for (int k = 0; k < 8; ++k) f[k] *= inv;
            ns_split<8>(f, h, l);
            nss_st(X, i, w, h);
            nss_st(X + xlo, i, w, l);
        }
        for (int step = 0; step < p.steps; ++step) {
            const float ca = p.coef[3 * step], cb = p.coef[3 * step + 1], cc = p.coef[3 * step + 2];
            run([&]() {
                product(acc_a, smem, smem, p.chunks, kc * 64, 0);
                if (p.terms == 3) {
                    product(acc_a, smem, smem + xlo, p.chunks, kc * 64, 1);
                    product(acc_a, smem + xlo, smem, p.chunks, kc * 64, 1);
                }
            });
            float* part = p.part + ((size_t)group * p.G + rank) * p.n * 128;
            for (int c = half * 16; c < p.n; c += 32) {
                uint32_t raw[16];
                __syncwarp();
                tmem_ld_x16(acc_a + c + ((uint32_t)(q * 32) << 16), raw);
                tmem_ld_wait();
                float v[16];
#pragma unroll
                for (int t = 0; t < 16; ++t) v[t] = __uint_as_float(raw[t]) * (1.f / (NS_SCALE * NS_SCALE));
                if (row >= p.n) continue;
                if (p.G > 1) {
#pragma unroll
                    for (int t = 0; t < 16; ++t)
                        if (c + t < p.n) part[(size_t)(c + t) * 128 + row] = v[t];
                } else {
#pragma unroll
                    for (int t = 0; t < 16; ++t)
                        if (c + t == row) {
                            sh.d[row] = v[t];
                            v[t] = 0.f;
                        }
                    uint32_t h[8], l[8];
                    ns_split<16>(v, h, l);
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        nss_st(E, row, c / 8 + w, h + 4 * w);
                        nss_st(E + elo, row, c / 8 + w, l + 4 * w);
                    }
                }
            }
            if (p.G > 1) {
                cluster_sync_all();
                // this CTA's columns j of A (rows j, A being symmetric): 8 entries a thread, summed in the CTAs' order, to everyone
                const int j0 = p.n * rank / p.G, j1 = p.n * (rank + 1) / p.G, n8 = (p.n + 7) / 8;
                const float* in = p.part + (size_t)group * p.G * p.n * 128;
                for (int u = threadIdx.x; u < (j1 - j0) * n8; u += NSS_THREADS) {
                    const int j = j0 + u / n8, w = u % n8;
                    alignas(32) float v[8];
                    float t[8];
                    ld8f(in + (size_t)j * 128 + w * 8, v);
#pragma unroll 4
                    for (int r = 1; r < p.G; ++r) {
                        ld8f(in + ((size_t)r * p.n + j) * 128 + w * 8, t);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] += t[k];
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (w * 8 + k == j)
                            for (int r = 0; r < p.G; ++r) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&sh.d[j]), r)), "f"(v[k]) : "memory");
                        if (w * 8 + k == j || w * 8 + k >= p.n) v[k] = 0.f;
                    }
                    uint32_t h[4], l[4];
                    ns_split<8>(v, h, l);
                    const uint32_t at = smem + e_at + nss_at(j, w);
                    for (int r = 0; r < p.G; ++r) {
                        nss_st_remote(at, r, h);
                        nss_st_remote(at + elo, r, l);
                    }
                }
                asm volatile("fence.proxy.async;" ::: "memory");
                cluster_sync_all();
            }
            const uint32_t ea = smem + e_at;
            run([&]() {
                product(acc_a, ea, ea, kc, kc * 64, 0);
                if (p.terms == 3) {
                    product(acc_a, ea, ea + elo, kc, kc * 64, 1);
                    product(acc_a, ea + elo, ea, kc, kc * 64, 1);
                }
            });
            const float di = sh.d[row];
            for (int c = half * 16; c < p.n; c += 32) {
                uint32_t raw[16], h[8], l[8];
                __syncwarp();
                tmem_ld_x16(acc_a + c + ((uint32_t)(q * 32) << 16), raw);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    nss_ld(E, row, c / 8 + w, h + 4 * w);
                    nss_ld(E + elo, row, c / 8 + w, l + 4 * w);
                }
                tmem_ld_wait();
                float v[16];
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    const float2 fh = half2_at(h[t / 2]), fl = half2_at(l[t / 2]);
                    const float e = t & 1 ? fh.y + fl.y : fh.x + fl.x, sq = __uint_as_float(raw[t]);
                    if (c + t == row && row < p.n) sh.rs[row] = ca + fmaf(cb, di, cc * fmaf(di, di, sq));
                    v[t] = c + t == row || c + t >= p.n ? 0.f : fmaf(cb, e, cc * fmaf(di + sh.d[c + t], e, sq));
                }
                if (row >= p.n) continue;
                ns_split<16>(v, h, l);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    nss_st(E, row, c / 8 + w, h + 4 * w);
                    nss_st(E + elo, row, c / 8 + w, l + 4 * w);
                }
            }
            run([&]() {
                // X lies with the contraction index (its rows) across: 16 rows a step, 64 columns a chunk
                const uint32_t idesc = (1u << 4) | ((uint32_t)(p.chunks * 8) << 17) | (8u << 24) | (1u << 16);
                uint32_t accumulate = 0;
                for (int t = 0; t < p.terms; ++t) {
                    const uint32_t fa = ea + (t == 2 ? elo : 0), xa = smem + (t == 1 ? xlo : 0);
                    for (int k = 0; k < 4 * kc; ++k) {
                        umma_bf16_lo<false>(acc_x, sdesc_lo(fa + (k >> 2) * NSS_CHUNK) + 2 * (k & 3), (((xa & 0x3FFFFu) >> 4) | ((NSS_CHUNK >> 4) << 16)) + k * 128, idesc, accumulate, 1u);
                        accumulate = 1;
                    }
                }
            });
            const float factor = sh.rs[row];
            for (int c = half * 16; c < p.chunks * 64; c += 32) {
                uint32_t raw[16], h[8], l[8];
                __syncwarp();
                tmem_ld_x16(acc_x + c + ((uint32_t)(q * 32) << 16), raw);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    nss_ld(X, row, c / 8 + w, h + 4 * w);
                    nss_ld(X + xlo, row, c / 8 + w, l + 4 * w);
                }
                tmem_ld_wait();
                if (row >= p.n) continue;
                float v[16];
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    const float2 fh = half2_at(h[t / 2]), fl = half2_at(l[t / 2]);
                    v[t] = fmaf(factor, t & 1 ? fh.y + fl.y : fh.x + fl.x, __uint_as_float(raw[t]));
                }
                ns_split<16>(v, h, l);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    nss_st(X, row, c / 8 + w, h + 4 * w);
                    nss_st(X + xlo, row, c / 8 + w, l + 4 * w);
                }
            }
        }
        __syncthreads();
        for (int u = threadIdx.x; u < p.n * units; u += NSS_THREADS) {
            const int i = p.in.tall ? u % p.n : u / units, w = p.in.tall ? u / p.n : u % units, c = c0 + w * 8;
            uint32_t h[4], l[4];
            float f[8];
            nss_ld(X, i, w, h);
            nss_ld(X + xlo, i, w, l);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 fh = half2_at(h[k]), fl = half2_at(l[k]);
                f[2 * k] = (fh.x + fl.x) * (1.f / NS_SCALE);
                f[2 * k + 1] = (fh.y + fl.y) * (1.f / NS_SCALE);
            }
            if (!p.in.tall && p.in.vec && c < p.m) {
                ns_put_o<8>(p.in, base + (size_t)i * p.in.cols + c, f);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < p.m) ns_put_o<1>(p.in, base + (p.in.tall ? (size_t)(c + k) * p.in.cols + i : (size_t)i * p.in.cols + c + k), f + k);
            }
        }
        __syncthreads();                        // X is read before the next matrix takes its place
    }
    if (sh.abort) {                             // products in flight end within microseconds; then the CTA may go
        const long long t0 = clock64();
        while (clock64() - t0 < 4000000) {}
    }
    tc_fence_before();
    meet();
    if (warp == 0) tmem_dealloc(tmem, 512);
}

static bool nss_attributes() {
    static PerDeviceFlag attr_set;
    if (attr_set.get()) return true;
    if (cudaFuncSetAttribute(ns_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NSS_SMEM) != cudaSuccess ||
        cudaFuncSetAttribute(ns_small_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    attr_set.set();
    return true;
}

// Clusters of `ctas` CTAs the device holds at a time.
static int nss_clusters(int ctas) {
    static std::atomic<int> known[64][5];
    int k = 0;
    while ((1 << k) < ctas) ++k;
    std::atomic<int>& slot = known[PerDeviceFlag::dev()][k];
    int n = slot.load(std::memory_order_relaxed);
    if (n) return n - 1;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(NSS_THREADS); cfg.dynamicSmemBytes = NSS_SMEM; cfg.attrs = attr; cfg.numAttrs = 1;
    if (!nss_attributes() || cudaOccupancyMaxActiveClusters(&n, ns_small_kernel, &cfg) != cudaSuccess || n < 0) {
        (void)cudaGetLastError();
        n = num_sms() / ctas;                   // no device to ask
    }
    slot.store(n + 1, std::memory_order_relaxed);
    return n;
}

NsSmallPlan ns_small_plan(int batch, int rows, int cols) {
    NsSmallPlan l = {};
    const int n = std::min(rows, cols), m = std::max(rows, cols), all = (m + 63) / 64;
    if (n > 128) return l;
    // As many CTAs as there are chunks of 64 columns (the slab's products and element-wise work get shorter, the exchange hardly
    // longer), fewer where a batch fills the device without.
    const int want = std::max(1, batch);
    for (int g = 16; g >= 1; g /= 2) {
        const int chunks = (all + g - 1) / g, clusters = nss_clusters(g);
        if ((g > all && g > 1) || clusters < 1) continue;
        if (chunks > NSS_MAX_CHUNKS) break;
        l.ctas = g;
        l.chunks = chunks;
        l.groups = std::min(want, clusters);
        if (clusters >= want) break;
    }
    l.terms = n <= 64 ? 3 : 1;
    l.bytes = l.ctas > 1 ? (size_t)l.groups * l.ctas * n * 128 * sizeof(float) : 256;
    return l;
}

int ns_small_run(const NsSmallPlan& plan, int batch, const NsInput& in, int steps, const float* coef, void* workspace, cudaStream_t stream) {
    NsSmall p = {};
    p.in = in;
    p.batch = batch; p.steps = steps; p.n = std::min(in.rows, in.cols); p.m = std::max(in.rows, in.cols);
    p.G = plan.ctas; p.groups = plan.groups; p.chunks = plan.chunks; p.terms = plan.terms;
    for (int i = 0; i < 3 * steps; ++i) p.coef[i] = coef[i];
    p.part = (float*)workspace;
    p.status = dev_status_ptr();
    if (!nss_attributes()) return DR_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.G; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(p.groups * p.G)); cfg.blockDim = dim3(NSS_THREADS); cfg.stream = stream;
    cfg.dynamicSmemBytes = NSS_SMEM;
    cfg.attrs = attr; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, ns_small_kernel, p) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
    count_launch();
    return launch_status();
}

}  // namespace dr
