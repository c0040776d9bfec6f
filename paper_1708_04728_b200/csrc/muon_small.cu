// The orthogonalised update of matrices with at most 128 rows (after transposing a tall one), a thread-block cluster per matrix.
//
// What bounds such a matrix is not its arithmetic but 15 dependent products, so nothing leaves the SM that does not have to.  A CTA
// keeps a slab of X's columns in shared memory for all steps, as float16 pairs in the layout that serves both as rows of X (A = X X^T,
// contraction along the slab) and as the second operand of F X.  Per step
//   A    each CTA multiplies its slab by its own transpose and leaves its part in global memory (L2); after a cluster barrier it sums the
//        columns it owns over all parts, in the CTAs' order, and after another one takes everyone's: 64 KB read twice at n = 128.
//        (Every CTA summing all parts for itself saves a barrier but took 7.5 us of a step with 8 CTAs; sending the sums to the
//        others' shared memory took longer than the round trip through L2.)
//   F    every CTA computes E E (E: A without its diagonal) and the polynomial for itself,
//   X    every CTA updates its slab in place.
// Products and element-wise terms as in the kernel for larger matrices (muon.cu); with few rows rounding errors average less, so
// matrices of up to 64 rows multiply hi hi + hi lo + lo hi: the tensor cores idle here either way (relative error of O 1e-6 .. 3e-5, 7e-5 for a single direction).
//
// Measured on a B200, five steps: 64 x 147 37 us (39 us with the optimiser's momentum and update), 128 x 864 58 us, 27 x 96 x 800 with the
// optimiser 72 us.  At 128 x 864 the tensor pipe is busy 5 % of the time and 41 % of the issue slots are taken: a step is a chain of
// element-wise passes over E and X (0.3 .. 0.9 us each) between three products of 0.7 .. 1.2 us from the barrier in front to the last MMA.
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "muon_common.cuh"

namespace dr {

constexpr int NSS_THREADS = 512;           // 16 warps: four share the 32 accumulator rows that each of them can read
constexpr int NSS_CHUNK = 128 * 128;        // 64 columns of 128 rows
constexpr int NSS_CHUNKS = 12;             // of shared memory: X (hi, lo) as wide as the slab, E (hi, lo) as wide as n
static_assert(NSS_CHUNKS * NSS_CHUNK + 1024 <= NS_SMEM_ALL, "");

struct NsSmall {
    NsInput in;
    int batch, steps, n, m, G, groups, chunks, terms;
    float coef[3 * DR_NS_MAX_STEPS];
    float* part;                // [group][CTA][column][128 rows]: parts of A
    uint4* sums;                // [group][row][8-column unit][hi, lo]: E
    float* diag;                // [group][128]
    int* status;
};

struct NsSmallShared {
    uint64_t done;
    uint32_t tmem_base;
    int abort;
    double red[NSS_THREADS / 32], norm[16];
    alignas(16) float d[128];
    float rs[128];
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
// and the same again 64 rows on
__device__ __forceinline__ void nss_st_rows(uint8_t* base, int row, int unit, const uint32_t* u, bool twice) {
    nss_st(base, row, unit, u);
    if (twice) nss_st(base + 64 * 128, row, unit, u);
}

// A CTA's slab in the user's memory, element by element (CN = 1) or, where rows are aligned and U is not tall, 8 columns at a time in 16-byte
// accesses.  Elements are taken as they lie in memory, across the ends of rows, so that every thread's rounds are full: row by row to
// the warps, the input of 64 x 147 took 6 us; like this 64 x 147 takes 39 instead of 43 us and 128 x 865 62 instead of 72.
struct NssPlace { int i, c, at; bool ok; };              // row and column in the slab, place in the user's matrix
template <int CN>
struct NssWalk {
    static constexpr int U = CN == 1 ? 10 : 2;              // places whose loads go out together
    int x, end, inner, start, skip;
    float inv;
    __device__ __forceinline__ NssWalk(const NsSmall& p, int c0) {
        const int width = max(min(p.m - c0, p.chunks * 64), 0);
        inner = CN == 8 ? p.chunks * 8 : p.in.tall ? p.n : width;
        x = threadIdx.x;
        end = CN == 8 ? p.n * inner : p.n * width;
        inv = 1.f / (float)inner;
        start = p.in.tall ? c0 * p.n : c0;
        skip = (p.in.tall ? p.n : p.in.cols) - inner;       // from one of the user's rows to the next (CN = 1)
    }
    __device__ __forceinline__ bool more() const { return x < end; }
    __device__ __forceinline__ void next() { x += U * NSS_THREADS; }
    __device__ __forceinline__ bool get(const NsSmall& p, int k, int c0, NssPlace& t) const {
        const int e = x + k * NSS_THREADS;
        // at most 32768 elements, rows of at most 256: the quotient is 0.5 / 256 or more from a whole number, its rounding error below 2^-15
        const int r = (int)(((float)e + 0.5f) * inv), y = e - r * inner;
        t.i = CN == 1 && p.in.tall ? y : r;
        t.c = CN == 1 && p.in.tall ? r : y * CN;
        t.at = start + (CN == 1 ? e + r * skip : t.i * p.in.cols + t.c);
        t.ok = e < end && c0 + t.c < p.m;
        return e < end;
    }
};
// v <- momentum v + g; U waits in the place of X, 16 bytes of a unit of 8 columns where its hi half goes and 16 where the lo half goes.
// Returns this thread's part of the sum of squares, in float64: no size of U overflows or vanishes.
template <int CN>
__device__ __forceinline__ double nss_load(const NsSmall& p, uint8_t* X, int xlo, int c0, size_t base) {
    constexpr int U = NssWalk<CN>::U;
    const NsInput& in = p.in;
    double s = 0.;
#pragma unroll 1
    for (NssWalk<CN> walk(p, c0); walk.more(); walk.next()) {
        alignas(16) float f[U][CN], v[U][CN];
        NssPlace t[U];
        bool mine[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            mine[k] = walk.get(p, k, c0, t[k]);
#pragma unroll
            for (int e = 0; e < CN; ++e) f[k][e] = v[k][e] = 0.f;
            if (!t[k].ok) continue;
            if (in.g_f32) ns_read<CN>((const float*)in.g + base + t[k].at, f[k]);
            else ns_read<CN>((const __nv_bfloat16*)in.g + base + t[k].at, f[k]);
            if (in.v) ns_read<CN>(in.v + base + t[k].at, v[k]);
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (in.v) {
#pragma unroll
                for (int e = 0; e < CN; ++e) v[k][e] = fmaf(in.momentum, v[k][e], f[k][e]);
                if (t[k].ok) ns_write<CN>(in.v + base + t[k].at, v[k]);
#pragma unroll
                for (int e = 0; e < CN; ++e) f[k][e] = in.nesterov ? fmaf(in.momentum, v[k][e], f[k][e]) : v[k][e];
            }
#pragma unroll
            for (int e = 0; e < CN; ++e) s = fma((double)f[k][e], (double)f[k][e], s);
            if (!mine[k]) continue;
            uint8_t* to = X + nss_at(t[k].i, t[k].c >> 3);
            if (CN == 8) {
                *reinterpret_cast<float4*>(to) = make_float4(f[k][0], f[k][1 % CN], f[k][2 % CN], f[k][3 % CN]);
                *reinterpret_cast<float4*>(to + xlo) = make_float4(f[k][4 % CN], f[k][5 % CN], f[k][6 % CN], f[k][7 % CN]);
            } else {
                *reinterpret_cast<float*>(to + (t[k].c & 4 ? xlo : 0) + (t[k].c & 3) * 4) = f[k][0];
            }
        }
    }
    return s;
}
template <int CN>
__device__ __forceinline__ void nss_store(const NsSmall& p, const uint8_t* X, int xlo, int c0, size_t base) {
    constexpr int U = NssWalk<CN>::U;
    const NsInput& in = p.in;
#pragma unroll 1
    for (NssWalk<CN> walk(p, c0); walk.more(); walk.next()) {
        float f[U][CN], w[U][CN];
        NssPlace t[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            walk.get(p, k, c0, t[k]);
            if (!t[k].ok) continue;
            if (in.w) ns_read<CN>(in.w + base + t[k].at, w[k]);
            const uint8_t* from = X + nss_at(t[k].i, t[k].c >> 3) + (CN == 1 ? (t[k].c & 7) * 2 : 0);
            if (CN == 8) {
                const uint4 h = *reinterpret_cast<const uint4*>(from), l = *reinterpret_cast<const uint4*>(from + xlo);
                const uint32_t hu[4] = {h.x, h.y, h.z, h.w}, lu[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                for (int e = 0; e < CN; ++e) {
                    const float2 fh = half2_at(hu[e / 2]), fl = half2_at(lu[e / 2]);
                    f[k][e] = (e & 1 ? fh.y + fl.y : fh.x + fl.x) * (1.f / NS_SCALE);
                }
            } else {
                f[k][0] = (__half2float(*reinterpret_cast<const __half*>(from)) + __half2float(*reinterpret_cast<const __half*>(from + xlo))) * (1.f / NS_SCALE);
            }
        }
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (!t[k].ok) continue;
            if (in.w) {
#pragma unroll
                for (int e = 0; e < CN; ++e) f[k][e] = fmaf(-in.lr_scale, f[k][e], in.keep * w[k][e]);
                ns_write<CN>(in.w + base + t[k].at, f[k]);
            }
            if (in.out) ns_write<CN>(in.out + base + t[k].at, f[k]);
        }
    }
}

// CN: how U is read and the result written, as in NssWalk (a kernel each: the registers of one for both cost every shape 2 to 4 us).
template <int CN>
__global__ void __launch_bounds__(NSS_THREADS, 1) ns_small_kernel(const __grid_constant__ NsSmall p) {
    extern __shared__ uint8_t nss_raw[];
    __shared__ NsSmallShared sh;
    if (cluster_lost(p.G, p.status)) return;
    const uint32_t smem = (smem_u32(nss_raw) + 1023u) & ~1023u;
    uint8_t* const X = nss_raw + (smem - smem_u32(nss_raw));           // hi chunks, then lo chunks
    const int xlo = p.chunks * NSS_CHUNK, e_at = 2 * xlo;
    const int kc = (p.n + 63) / 64, elo = kc * NSS_CHUNK;              // chunks of an n x n operand
    uint8_t* const E = X + e_at;                                       // E, later F: hi, then lo
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    // A warp reads 32 of the accumulators' 128 rows, and warps whose rows are the same modulo 128 share a quarter of the SM.  Matrices of up to 64
    // rows fill only half of that, so theirs are held twice, as rows 0 .. 63 and 64 .. 127 of the first operands: all warps have rows, and
    // half as many columns of them (64 x 147: 47 -> 41 us, then).
    const bool twice = p.n <= 64;
    const int q = warp & 3, row = (twice ? q & 1 : q) * 32 + lane;
    const int first = ((warp >> 2) + (twice ? q >> 1 << 2 : 0)) * 8, stride = twice ? 64 : 32;      // a warp's columns: 8 from here, 8 a stride on
    const bool has_rows = row - lane < p.n;
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
#pragma unroll 1
        for (int k = 0; k < kchunks; ++k, pa += NSS_CHUNK, qa += NSS_CHUNK)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                umma_bf16_lo<false>(d, sdesc_lo(pa) + 2 * s, sdesc_lo(qa) + 2 * s, idesc, accumulate, 1u);
                accumulate = 1;
            }
    };

    for (int b = group; b < p.batch; b += p.groups) {
        const size_t base = (size_t)b * p.n * p.m;
        if (CN == 1 && b != group) {   // columns past m: zero again, whatever the matrix before left there
            for (int i = threadIdx.x; i < p.n * units; i += NSS_THREADS) {
                const int r = i / units, w = i - r * units;
                const uint32_t zero[4] = {0, 0, 0, 0};
                if (c0 + w * 8 + 8 <= p.m) continue;
                nss_st(X, r, w, zero);
                nss_st(X + xlo, r, w, zero);
            }
            __syncthreads();
        }
        double s = nss_load<CN>(p, X, xlo, c0, base);
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
        const NsFactor by = ns_factor(s, p.in.eps);
#pragma unroll 1
        for (int u = threadIdx.x; u < p.n * units; u += NSS_THREADS) {
            const int i = u / units, w = u - i * units;
            uint32_t h[4], l[4];
            float f[8];
            nss_ld(X, i, w, h);
            nss_ld(X + xlo, i, w, l);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                f[k] = __uint_as_float(h[k]) * by.first * by.second;
                f[4 + k] = __uint_as_float(l[k]) * by.first * by.second;
            }
            ns_split<8>(f, h, l);
            nss_st_rows(X, i, w, h, twice);
            nss_st_rows(X + xlo, i, w, l, twice);
        }
        for (int step = 0; step < p.steps; ++step) {
            const float ca = p.coef[3 * step], cb = p.coef[3 * step + 1], cc = p.coef[3 * step + 2];
            run([&]() {
#pragma unroll 1
                for (int t = 0; t < p.terms; ++t) product(acc_a, smem + (t == 2 ? xlo : 0), smem + (t == 1 ? xlo : 0), p.chunks, kc * 64, t > 0);
            });
            float* const part = p.part + (size_t)group * p.G * p.n * 128;
            if (has_rows)
#pragma unroll 1
                for (int c = first; c < p.n; c += stride) {
                    uint32_t raw[8];
                    __syncwarp();
                    tmem_ld_x8(acc_a + c + ((uint32_t)(q * 32) << 16), raw);
                    tmem_ld_wait();
                    float v[8];
#pragma unroll
                    for (int t = 0; t < 8; ++t) v[t] = __uint_as_float(raw[t]) * (1.f / (NS_SCALE * NS_SCALE));
                    if (p.G > 1) {
#pragma unroll
                        for (int t = 0; t < 8; ++t)
                            if (c + t < p.n) part[(size_t)rank * p.n * 128 + (c + t) * 128 + row] = v[t];
                    } else if (row < p.n) {
                        float d = 0.f;
#pragma unroll
                        for (int t = 0; t < 8; ++t) {
                            d = c + t == row ? v[t] : d;
                            v[t] = c + t == row ? 0.f : v[t];
                        }
                        if (row >= c && row < c + 8) sh.d[row] = d;
                        uint32_t h[4], l[4];
                        ns_split<8>(v, h, l);
                        nss_st_rows(E, row, c / 8, h, twice);
                        nss_st_rows(E + elo, row, c / 8, l, twice);
                    }
                }
            if (p.G > 1) {
                cluster_sync_all();
                const int j0 = p.n * rank / p.G, j1 = p.n * (rank + 1) / p.G, n8 = (p.n + 7) / 8;
                uint4* const sums = p.sums + (size_t)group * p.n * n8 * 2;
                float* const diag = p.diag + (size_t)group * 128;
#pragma unroll 1
                for (int u = threadIdx.x; u < (j1 - j0) * n8; u += NSS_THREADS) {
                    const int jj = u / n8, j = j0 + jj, w = u - jj * n8;
                    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, t[8];
                    const float* from = part + j * 128 + w * 8;
#pragma unroll 8
                    for (int r = 0; r < p.G; ++r, from += p.n * 128) {
                        ld8f(from, t);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[k] += t[k];
                    }
                    float d = 0.f;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        d = w * 8 + k == j ? v[k] : d;
                        v[k] = w * 8 + k == j || w * 8 + k >= p.n ? 0.f : v[k];
                    }
                    if ((j >> 3) == w) diag[j] = d;
                    uint32_t h[4], l[4];
                    ns_split<8>(v, h, l);
                    sums[(j * n8 + w) * 2] = make_uint4(h[0], h[1], h[2], h[3]);
                    sums[(j * n8 + w) * 2 + 1] = make_uint4(l[0], l[1], l[2], l[3]);
                }
                cluster_sync_all();
                if (threadIdx.x < p.n) sh.d[threadIdx.x] = diag[threadIdx.x];
#pragma unroll 4
                for (int u = threadIdx.x; u < p.n * n8 * 2; u += NSS_THREADS) {
                    const int j = u / (n8 * 2), w = u - j * (n8 * 2);
                    const uint4 v = sums[u];
                    uint8_t* const to = E + (w & 1 ? elo : 0) + nss_at(j, w >> 1);
                    *reinterpret_cast<uint4*>(to) = v;
                    if (twice) *reinterpret_cast<uint4*>(to + 64 * 128) = v;
                }
            }
            // E E, then F X; either product updates pairs in shared memory in place: E -> F = (b + c (d_i + d_j)) E + c E E, X -> r X + F X.
            // One code for both: a step's instructions are fetched once per step, and the fetch shows.
            const uint32_t ea = smem + e_at;
#pragma unroll 1
            for (int pass = 0; pass < 2; ++pass) {
                const bool is_x = pass;
                run([&]() {
                    const uint32_t idesc = (1u << 4) | ((uint32_t)(is_x ? p.chunks * 8 : kc * 8) << 17) | (8u << 24) | (is_x ? 1u << 16 : 0u);
                    const uint32_t d = is_x ? acc_x : acc_a, qh = is_x ? smem : ea, ql = is_x ? smem + xlo : ea + elo;
                    uint32_t accumulate = 0;
#pragma unroll 1
                    for (int t = 0; t < p.terms; ++t) {
                        const uint32_t fa = ea + (t == 2 ? elo : 0), xa = t == 1 ? ql : qh;
#pragma unroll 1
                        for (int k = 0; k < 4 * kc; ++k) {
                            // X lies with the contraction index (its rows) across: 16 rows a step, 64 columns a chunk
                            const uint32_t bd = is_x ? (((xa & 0x3FFFFu) >> 4) | ((NSS_CHUNK >> 4) << 16)) + k * 128 : sdesc_lo(xa + (k >> 2) * NSS_CHUNK) + 2 * (k & 3);
                            umma_bf16_lo<false>(d, sdesc_lo(fa + (k >> 2) * NSS_CHUNK) + 2 * (k & 3), bd, idesc, accumulate, 1u);
                            accumulate = 1;
                        }
                    }
                });
                if (!has_rows) continue;
                const float di = sh.d[row], factor = is_x ? sh.rs[row] : fmaf(cc, di, cb), fd = is_x ? 0.f : cc, beta = is_x ? 1.f : cc;
                uint8_t* const at = is_x ? X : E;
                const int lo = is_x ? xlo : elo, width = is_x ? p.chunks * 64 : p.n;
                const uint32_t acc = (is_x ? acc_x : acc_a) + ((uint32_t)(q * 32) << 16);
#pragma unroll 1
                for (int c = first; c < width; c += stride) {
                    uint32_t raw[8], h[4], l[4];
                    __syncwarp();
                    tmem_ld_x8(acc + c, raw);
                    nss_ld(at, row, c / 8, h);
                    nss_ld(at + lo, row, c / 8, l);
                    float dj[8], v[8];
#pragma unroll
                    for (int t = 0; t < 8; t += 4) {
                        const float4 x = *reinterpret_cast<const float4*>(&sh.d[(c & 127) + t]);
                        dj[t] = x.x; dj[t + 1] = x.y; dj[t + 2] = x.z; dj[t + 3] = x.w;
                    }
                    tmem_ld_wait();
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        const float2 fh = half2_at(h[t / 2]), fl = half2_at(l[t / 2]);
                        v[t] = fmaf(is_x ? factor : fmaf(fd, dj[t], factor), t & 1 ? fh.y + fl.y : fh.x + fl.x, beta * __uint_as_float(raw[t]));
                    }
                    if (!is_x) {                // selects, one store: branches of one lane each took 1.3 us a step
                        float sq = 0.f;
#pragma unroll
                        for (int t = 0; t < 8; ++t) {
                            sq = c + t == row ? __uint_as_float(raw[t]) : sq;
                            v[t] = c + t == row || c + t >= p.n ? 0.f : v[t];
                        }
                        if (row >= c && row < c + 8 && row < p.n) sh.rs[row] = ca + fmaf(cb, di, cc * fmaf(di, di, sq));
                    }
                    if (row < p.n) {
                        ns_split<8>(v, h, l);
                        nss_st_rows(at, row, c / 8, h, twice);
                        nss_st_rows(at + lo, row, c / 8, l, twice);
                    }
                }
            }
        }
        __syncthreads();
        nss_store<CN>(p, X, xlo, c0, base);
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

typedef void (*NssKernel)(const NsSmall);
static bool nss_attributes() {
    static PerDeviceFlag attr_set;
    if (attr_set.get()) return true;
    for (NssKernel k : {ns_small_kernel<8>, ns_small_kernel<1>})
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, NS_SMEM_ALL) != cudaSuccess ||
            cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
            (void)cudaGetLastError();
            return false;
        }
    attr_set.set();
    return true;
}

int ns_small_lost_cluster(cudaStream_t stream) {
    NsSmall p = {};
    p.G = 2;
    p.status = dev_status_ptr();
    if (!nss_attributes()) return DR_ERR_CUDA;
    ns_small_kernel<8><<<2, NSS_THREADS, NS_SMEM_ALL, stream>>>(p);
    count_launch();
    return launch_status();
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
    cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(NSS_THREADS); cfg.dynamicSmemBytes = NS_SMEM_ALL; cfg.attrs = attr; cfg.numAttrs = 1;
    if (!nss_attributes() || cudaOccupancyMaxActiveClusters(&n, ns_small_kernel<8>, &cfg) != cudaSuccess || n < 0) {
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
    // One CTA where it holds X: no exchange.  Otherwise a chunk of 64 columns each, more where a batch would not fit the device
    // (128 x 864, at an earlier stage: 60 us with 16 CTAs, 64 with 8, 76 with 4).
    for (int g = 1; g <= 16; g *= 2) {
        const int chunks = (all + g - 1) / g, clusters = nss_clusters(g);
        if (chunks > 4 || 2 * chunks + 2 * ((n + 63) / 64) > NSS_CHUNKS || clusters < 1) continue;
        if (l.ctas && clusters < std::max(1, batch)) break;
        l.ctas = g;
        l.chunks = chunks;
        l.groups = std::min(std::max(1, batch), clusters);
        if (g == 1 || chunks == 1) break;
    }
    l.terms = n <= 64 ? 3 : 1;
    size_t at = 0;
    auto take = [&](size_t& where, size_t bytes) { where = at; at += (bytes + 255) / 256 * 256; };
    take(l.part, l.ctas > 1 ? (size_t)l.groups * l.ctas * n * 128 * sizeof(float) : 0);
    take(l.sums, l.ctas > 1 ? (size_t)l.groups * n * ((n + 7) / 8) * 2 * sizeof(uint4) : 0);
    take(l.diag, (size_t)l.groups * 128 * sizeof(float));
    l.bytes = at;
    return l;
}

int ns_small_run(const NsSmallPlan& plan, int batch, const NsInput& in, int steps, const float* coef, void* workspace, cudaStream_t stream) {
    NsSmall p = {};
    p.in = in;
    p.batch = batch; p.steps = steps; p.n = std::min(in.rows, in.cols); p.m = std::max(in.rows, in.cols);
    p.G = plan.ctas; p.groups = plan.groups; p.chunks = plan.chunks; p.terms = plan.terms;
    for (int i = 0; i < 3 * steps; ++i) p.coef[i] = coef[i];
    p.part = (float*)((char*)workspace + plan.part);
    p.sums = (uint4*)((char*)workspace + plan.sums);
    p.diag = (float*)((char*)workspace + plan.diag);
    p.status = dev_status_ptr();
    if (!nss_attributes()) return DR_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = p.G; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3((unsigned)(p.groups * p.G)); cfg.blockDim = dim3(NSS_THREADS); cfg.stream = stream;
    cfg.dynamicSmemBytes = NS_SMEM_ALL;
    cfg.attrs = attr; cfg.numAttrs = 1;
    const NssKernel kernel = in.vec && !in.tall ? ns_small_kernel<8> : ns_small_kernel<1>;
    if (cudaLaunchKernelEx(&cfg, kernel, p) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
    count_launch();
    return launch_status();
}

}  // namespace dr
