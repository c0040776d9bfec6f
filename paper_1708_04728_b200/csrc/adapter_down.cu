// The adapters' first product, out[m][r] = factor * sum_l D(z)[m][l] f_a[r][l] with a the adapter of row m: few columns, so it is bound
// by the bytes of z (and, for single rows, of f).  Warps multiply fragments (mma.sync) that they load straight from memory: the order of l
// within a product is free, so a thread takes 16 consecutive l of its rows with 16-byte loads and its values of four MMAs lie in its own
// registers; no shared memory, and the dropout's mask is drawn where the values are.  A warp whose rows belong to several adapters does
// the product once for each and keeps the rows that are that adapter's.
//
// Few rows: the warps of a CTA share 16 rows and split l, a cluster of CTAs takes ranges of l (their sums meet in distributed shared memory, in
// order), and further clusters take adapters of their own.
#include <algorithm>

#include "adapter.cuh"
#include "umma_ptx.cuh"

namespace dr {

struct DownParams {
    AdRows rows;
    int L, L8, R, Rp, ks, zsplit;
    int l_range;                // l of a CTA's range, a multiple of 64
    const __nv_bfloat16 *z, *f;
    size_t ldz, ldf;
    DropKey key;
    float factor, after;
    const float* scale;
    int terms;
    __nv_bfloat16* out;
    float* keep;
    int* row_id;
};

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// MT tiles of 16 rows, RT tiles of 8 columns a warp; JOIN: the 8 warps of a CTA split l over the same rows, else each has rows of its own
template <int MT, int RT, bool DROP, bool JOIN>
__global__ void __launch_bounds__(256) adapter_down_kernel(const DownParams p) {
    __shared__ float join[JOIN ? 8 : 1][JOIN ? 16 : 1][JOIN ? RT * 8 + 2 : 1];
    __shared__ alignas(8) float range[JOIN ? 16 * RT * 8 : 1];              // this range's sums, read by the cluster
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, q = lane & 3;
    const int m0 = ((int)blockIdx.x * (JOIN ? 1 : 8) + (JOIN ? 0 : warp)) * MT * 16;
    const int ks = blockIdx.y, zi = (int)blockIdx.z % p.zsplit, r0 = ((int)blockIdx.z / p.zsplit) * RT * 8;
    const int l0 = ks * p.l_range, l1 = min(p.L8, l0 + p.l_range);
    if (m0 >= p.rows.M) return;                                  // JOIN: the whole CTA
    // z on its way to L2 while the rows' adapters are looked up: a line a thread
    for (int i = JOIN ? (int)threadIdx.x : lane; i < MT * 16 * ((l1 - l0 + 63) >> 6); i += JOIN ? 256 : 32) {
        const int row = i % (MT * 16), l = l0 + 64 * (i / (MT * 16));
        if (m0 + row < p.rows.M && l < l1) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.z + (size_t)(m0 + row) * p.ldz + l));
    }
    int id = adapter_of_warp_row(p.rows, m0, lane);
    if (lane >= MT * 16) id = ROW_NONE;
    else if (p.row_id && blockIdx.y == 0 && blockIdx.z == 0 && (!JOIN || warp == 0) && m0 + lane < p.rows.M) p.row_id[m0 + lane] = id;
    const unsigned long long off = DROP ? drop_offset(p.key) : 0ull;

    const __nv_bfloat16* zr[MT][2];
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) zr[t][h] = p.z + (size_t)min(m0 + 16 * t + 8 * h + g, p.rows.M - 1) * p.ldz;

    // t of a row of this warp's at two neighbouring columns (the first even)
    auto put = [&](int row, int r, float x, float y, float scale) {
        if (p.keep) {
            float* to = p.keep + (size_t)(m0 + row) * p.R + r;
            if (r < p.R) to[0] = x;
            if (r + 1 < p.R) to[1] = y;
        }
        uint32_t u[3];
        split3(x * scale, y * scale, u[0], u[1], u[2]);
        uint32_t* to = reinterpret_cast<uint32_t*>(p.out + (size_t)(m0 + row) * p.terms * p.Rp + r);
        to[0] = u[0];
        to[p.Rp >> 1] = u[1];
        if (p.terms == 3) to[p.Rp] = u[2];
    };
    if (p.keep && id == ROW_SHARED && blockIdx.y == 0 && zi == 0 && (!JOIN || warp == 0))
        for (int r = r0; r < min(p.R, r0 + RT * 8); ++r) p.keep[(size_t)(m0 + lane) * p.R + r] = 0.f;
    int number = 0;
    for (unsigned rest = __ballot_sync(0xffffffffu, id >= 0); rest;) {
        const int a = __shfl_sync(0xffffffffu, id, __ffs(rest) - 1);
        const unsigned mine = __ballot_sync(0xffffffffu, id == a);
        rest &= ~mine;
        if (number++ % p.zsplit != zi) continue;
        const float scale = (p.scale ? __ldg(p.scale + a) : 1.f) * p.after;
        float acc[MT][RT][4] = {};
        const __nv_bfloat16* f = p.f + ((size_t)a * p.R + r0 + g) * p.ldf;
#pragma unroll 1
        for (int l = l0 + (JOIN ? warp * 64 : 0); l < l1; l += JOIN ? 512 : 64) {
            uint32_t zw[MT][2][8], fw[RT][8];
            const int lq = l + 16 * q;
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (lq + 8 * k < l1) v = __ldg(reinterpret_cast<const uint4*>(zr[t][h] + lq + 8 * k));
                        zw[t][h][4 * k] = v.x; zw[t][h][4 * k + 1] = v.y; zw[t][h][4 * k + 2] = v.z; zw[t][h][4 * k + 3] = v.w;
                    }
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (r0 + 8 * r + g < p.R && lq + 8 * k < l1) v = __ldg(reinterpret_cast<const uint4*>(f + (size_t)8 * r * p.ldf + lq + 8 * k));
                    fw[r][4 * k] = v.x; fw[r][4 * k + 1] = v.y; fw[r][4 * k + 2] = v.z; fw[r][4 * k + 3] = v.w;
                }
            if (DROP) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const unsigned long long e = (unsigned long long)(m0 + 16 * t + 8 * h + g) * p.L + lq + 8 * k;
                            const uint32_t bits = drop_bits8_at(p.key, off, e);
                            const uint4 v = drop_apply8(make_uint4(zw[t][h][4 * k], zw[t][h][4 * k + 1], zw[t][h][4 * k + 2], zw[t][h][4 * k + 3]), bits);
                            zw[t][h][4 * k] = v.x; zw[t][h][4 * k + 1] = v.y; zw[t][h][4 * k + 2] = v.z; zw[t][h][4 * k + 3] = v.w;
                        }
            }
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int r = 0; r < RT; ++r)
                        mma_bf16(acc[t][r], zw[t][0][2 * s], zw[t][1][2 * s], zw[t][0][2 * s + 1], zw[t][1][2 * s + 1], fw[r][2 * s], fw[r][2 * s + 1]);
        }
        if (JOIN) {
#pragma unroll
            for (int t = 0; t < MT; ++t) {
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) join[warp][8 * (i >> 1) + g][8 * r + 2 * q + (i & 1)] = acc[t][r][i];
                __syncthreads();
                const int row = threadIdx.x >> 4, col = 2 * (threadIdx.x & 15);        // 16 threads to a row, two columns each
                const bool keeps = mine >> (16 * t + row) & 1;
#pragma unroll 1
                for (int r = col; r < RT * 8; r += 32) {
                    float x = 0.f, y = 0.f;
#pragma unroll
                    for (int w = 0; w < 8; ++w) { x += join[w][row][r]; y += join[w][row][r + 1]; }
                    if (p.ks > 1) { range[row * RT * 8 + r] = x; range[row * RT * 8 + r + 1] = y; }
                    else if (keeps && r0 + r < p.Rp) put(16 * t + row, r0 + r, x * p.factor, y * p.factor, scale);
                }
                if (p.ks > 1) {
                    ptx::cluster_sync_all();
#pragma unroll 1
                    for (int r = col; r < RT * 8; r += 32) {
                        if (row % p.ks != ks) continue;          // the cluster's CTAs share the rows
                        float x = 0.f, y = 0.f;
                        for (int k = 0; k < p.ks; ++k) {
                            float u, v;
                            asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(u), "=f"(v) : "r"(ptx::mapa_shared(ptx::smem_u32(range + row * RT * 8 + r), (uint32_t)k)) : "memory");
                            x += u; y += v;
                        }
                        if (keeps && r0 + r < p.Rp) put(16 * t + row, r0 + r, x * p.factor, y * p.factor, scale);
                    }
                    ptx::cluster_sync_all();                     // the sums are read: they may be overwritten, the CTA may leave
                } else {
                    __syncthreads();
                }
            }
        } else {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = 16 * t + 8 * h + g, c = r0 + 8 * r + 2 * q;
                        if ((mine >> row & 1) && c < p.Rp) put(row, c, acc[t][r][2 * h] * p.factor, acc[t][r][2 * h + 1] * p.factor, scale);
                    }
        }
    }
}

DownPlan adapter_down_plan(int M, int L, int R, int adapters, int segments) {
    DownPlan d = {};
    d.rt = R <= 8 ? 1 : R <= 16 ? 2 : R <= 32 ? 4 : 8;
    d.rchunks = (R + 8 * d.rt - 1) / (8 * d.rt);
    const int sms = num_sms();
    d.ks = d.zsplit = 1;
    if (M > 256ll * sms) {                  // a warp to every 32 rows fills the device
        d.mt = 2; d.warps_k = 1; d.rows_cta = 256;
        return d;
    }
    d.mt = M > 32 * sms ? 2 : 1;
    d.warps_k = 8; d.rows_cta = 16 * d.mt;
    const int tiles = (M + d.rows_cta - 1) / d.rows_cta;
    if (tiles < sms) {
        d.ks = std::max(1, std::min(std::min(8, (L + 511) / 512), 2 * sms / tiles));     // 8: the largest cluster every device holds
        const int distinct = std::min(std::min(16, M), std::min(adapters, segments));
        d.zsplit = std::max(1, std::min(distinct, 4 * sms / (tiles * d.ks)));
    }
    return d;
}

template <int MT, int RT, bool JOIN>
static int down_launch(const DownPlan& d, const DownParams& p, cudaStream_t s) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((p.rows.M + d.rows_cta - 1) / d.rows_cta), (unsigned)d.ks, (unsigned)(d.zsplit * d.rchunks));
    cfg.blockDim = dim3(256);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = 1; attr[0].val.clusterDim.y = (unsigned)d.ks; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = d.ks > 1 ? 1 : 0;
    const cudaError_t e = p.key.thr ? cudaLaunchKernelEx(&cfg, adapter_down_kernel<MT, RT, true, JOIN>, p) : cudaLaunchKernelEx(&cfg, adapter_down_kernel<MT, RT, false, JOIN>, p);
    if (e != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
    count_launch();
    return DR_OK;
}
template <int RT>
static int down_launch_rt(const DownPlan& d, const DownParams& p, cudaStream_t s) {
    if (d.warps_k == 1) return down_launch<2, RT, false>(d, p, s);
    return d.mt == 2 ? down_launch<2, RT, true>(d, p, s) : down_launch<1, RT, true>(d, p, s);
}

int adapter_down_run(const DownPlan& d, const AdRows& rows, int L, int R, int Rp, const __nv_bfloat16* z, size_t ldz, const __nv_bfloat16* f, size_t ldf,
                     const DropKey& key, float factor, const float* scale, float after, int terms, __nv_bfloat16* out, float* keep, int* row_id, cudaStream_t s) {
    DownParams p;
    p.rows = rows;
    p.L = L; p.L8 = (L + 7) / 8 * 8; p.R = R; p.Rp = Rp; p.ks = d.ks; p.zsplit = d.zsplit;
    p.l_range = (((L + d.ks - 1) / d.ks) + 63) / 64 * 64;
    p.z = z; p.f = f; p.ldz = ldz; p.ldf = ldf;
    p.key = key; p.factor = factor; p.scale = scale; p.after = after; p.terms = terms; p.out = out; p.keep = keep; p.row_id = row_id;
    if (d.rt == 1) return down_launch_rt<1>(d, p, s);
    if (d.rt == 2) return down_launch_rt<2>(d, p, s);
    return d.rt == 4 ? down_launch_rt<4>(d, p, s) : down_launch_rt<8>(d, p, s);
}

// ---- layouts ------------------------------------------------------------------------------------------------------
__global__ void adapter_align_kernel(size_t rows, int cols, const __nv_bfloat16* __restrict__ src, size_t ld, __nv_bfloat16* __restrict__ dst, size_t ldd) {
    const size_t row = (size_t)blockIdx.x * blockDim.y + threadIdx.y;
    if (row >= rows) return;
    for (int c = 2 * (int)threadIdx.x; c < (int)ldd; c += 64) {
        __nv_bfloat162 v;
        v.x = c < cols ? src[row * ld + c] : __float2bfloat16_rn(0.f);
        v.y = c + 1 < cols ? src[row * ld + c + 1] : __float2bfloat16_rn(0.f);
        *reinterpret_cast<__nv_bfloat162*>(dst + row * ldd + c) = v;
    }
}
int adapter_align_run(size_t rows, int cols, const __nv_bfloat16* src, size_t ld, __nv_bfloat16* dst, size_t ldd, cudaStream_t s) {
    adapter_align_kernel<<<(unsigned)((rows + 7) / 8), dim3(32, 8), 0, s>>>(rows, cols, src, ld, dst, ldd);
    count_launch();
    return launch_status();
}

}  // namespace dr
