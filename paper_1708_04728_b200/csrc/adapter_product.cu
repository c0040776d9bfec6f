// The shared product with the adapters' second factors in the same accumulator, on the tensor cores (tcgen05, accumulators in TMEM):
//   out[m][c] = act(sum_l z[m][l] w[c][l] + bias[c] + sum_r T[m][r] f_a[c][r]),   T = scale_a factor t,  a the adapter of row m.
//
// A tile of 128 rows (256 by a pair of CTAs) may hold rows of many adapters.  Behind the blocks of 64 l it takes further
// blocks for the adapters in use among its rows, each with `rank` columns of its own: a row has its T in its adapter's columns and zeros in
// the others', so the same MMAs serve any mixture of requests, and the work grows with the adapters' bytes, which have to be read anyway.  T
// enters as the sum of two bfloat16 values (its columns twice, high and low), because a single one would cost the adapter's part 2^-9; of three
// where the result is float32.
// Where a mask lies between the adapter's product and the sum (the gradient of the input behind a dropout), that product has an accumulator of its own
// and the drain draws the mask again.
//
// 0 * inf is NaN: entries of f that are not finite are left out of these blocks and added, for the rows of their own adapter only, in
// the drain.
//
// 12 warps: 0 loads (TMA), 1 issues MMAs, 4-7 drain, 8-11 find the rows' adapters and build the further blocks in the ring's stages.
#include <algorithm>

#include "adapter.cuh"
#include "conv_common.cuh"
#include "umma_ptx.cuh"

namespace dr {
using namespace ptx;

constexpr int AP_THREADS = 384;
constexpr int AP_MAX_STAGES = 16;
constexpr int AP_SMEM = 200 * 1024;
constexpr int AP_TILE = 128;
constexpr int AP_CACHE = 32 * 1024;     // T of a tile of few rows

struct ApParams {
    AdRows rows;
    int L, C, R, Rp;
    int terms, width;           // bfloat16 values to a T, columns of T in a further block of 64: 2 and 32, 3 and 16
    int nt;                     // columns of a tile
    int tiles_c, tiles;
    int kblocks, kpb, main_stages, stages;
    uint32_t a_bytes, b_bytes, stage_bytes;     // of a block of 64 l: z rows, w of this CTA; of a stage
    uint32_t acc_cols, tmem_cols;
    const int* row_id;          // nullptr: found here, ahead of the kernel in front (few rows)
    int cache;                  // bytes of T kept in shared memory, or 0
    const float *t, *scale, *bias;
    const __nv_bfloat16* f;
    size_t ldf;
    int f_vec;
    float factor;
    float* keep;
    unsigned flags;
    void* out;
    size_t ldo;
    int out_vec;                // rows of the output on 16-byte boundaries
    DropKey key;
    int* status;
};

struct ApShared {
    uint64_t full[AP_MAX_STAGES], empty[AP_MAX_STAGES], tfull[2], tempty[2], ifull[2], iempty[2], loads[2], built[2];
    uint32_t tmem;
    int abort;
    int ext[2];                 // columns of T of the tile
    int odd[2];                 // number (from 1) of the latest tile that met an f that is not finite
    int slot[2][AP_TILE];       // place of the row's adapter in list, ROW_SHARED or ROW_NONE
    uint16_t list[2][2 * AP_TILE];
    uint32_t bits[128];
    int before[128];
    int sums[4];
    float bias[4][256];
};

__device__ __forceinline__ uint32_t sdesc_rows_lo(uint32_t smem_addr, uint32_t box) {    // contraction index = row of a 64-column box
    return ((smem_addr & 0x3FFFFu) >> 4) | (((box >> 4) & 0x3FFFu) << 16);
}
__device__ __forceinline__ void builders_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
// the same, and whether any of them says so: they leave together or not at all, since this barrier has no limit
__device__ __forceinline__ bool builders_any(bool v) {
    uint32_t r;
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 q, %1, 0;\nbar.red.or.pred p, 1, 128, q;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(r) : "r"((uint32_t)v) : "memory");
    return r != 0;
}
__device__ __forceinline__ void st_shared16(uint32_t addr, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// entries that are not finite become zero; true if there was one
__device__ __forceinline__ bool finite_only(uint4& v) {
    bool any = false;
    uint32_t* u = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t l = (u[i] & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u, h = (u[i] & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u;
        any |= (l | h) != 0;
        u[i] &= ~(l | h);
    }
    return any;
}
// stages that hold the further blocks of `ext` columns
__device__ __forceinline__ int further_stages(const ApParams& p, int ext) {
    const int blocks = (ext + p.width - 1) / p.width;
    return (blocks + p.kpb - 1) / p.kpb;
}
// eight T as bfloat16 values
template <int TERMS>
__device__ __forceinline__ void split8(const float* v, float c, uint4* o) {
    uint32_t u[3][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (TERMS == 2) split2(v[2 * i] * c, v[2 * i + 1] * c, u[0][i], u[1][i]);
        else split3(v[2 * i] * c, v[2 * i + 1] * c, u[0][i], u[1][i], u[2][i]);
    }
#pragma unroll
    for (int k = 0; k < TERMS; ++k) o[k] = make_uint4(u[k][0], u[k][1], u[k][2], u[k][3]);
}

// PAIR: tiles of 256 rows by two CTAs.  ROWS: w and f have the contraction index as their rows.  DUAL: an accumulator of its own for the adapters.
// TERMS: bfloat16 values to a T.
template <bool PAIR, bool ROWS, bool DUAL, int TERMS>
__global__ void __launch_bounds__(AP_THREADS, 1)
adapter_product_kernel(const __grid_constant__ CUtensorMap map_z, const __grid_constant__ CUtensorMap map_w, const ApParams p) {
    extern __shared__ uint8_t ap_raw[];
    __shared__ ApShared sh;
    const uint32_t ring = (smem_u32(ap_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const int unit = PAIR ? (int)blockIdx.x >> 1 : (int)blockIdx.x, units = PAIR ? (int)gridDim.x >> 1 : (int)gridDim.x;
    const int tile_m = PAIR ? 2 * AP_TILE : AP_TILE;
    const int cols = PAIR ? p.nt >> 1 : p.nt;                  // columns of w that this CTA loads
    volatile int* abort_flag = &sh.abort;
    constexpr int WIDTH = TERMS == 2 ? 32 : 16;
    // after the ring, 4 KB for each draining warp, and T of a tile of few rows
    const uint32_t stage_out = ring + (uint32_t)p.stages * p.stage_bytes + (p.a_bytes < 16384u ? 16384u - p.a_bytes : 0u);
    float* const cache = reinterpret_cast<float*>(ap_raw + (stage_out + 4 * 4096u - smem_u32(ap_raw)));

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { mbar_init(&sh.full[i], PAIR ? 2 : 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.tfull[i], 1);
            mbar_init(&sh.tempty[i], PAIR ? 8 : 4);
            mbar_init(&sh.loads[i], 1);
            mbar_init(&sh.built[i], 1);
            mbar_init(&sh.ifull[i], 128);
            mbar_init(&sh.iempty[i], 5 + (rank == 0 ? 1 : 0));
        }
        sh.abort = 0;
        sh.odd[0] = sh.odd[1] = 0;
        fence_barrier_init();
        prefetch_tensormap(&map_z);
        prefetch_tensormap(&map_w);
    }
    if (warp == 1) {
        if (PAIR) { tmem_alloc_pair(&sh.tmem, p.tmem_cols); tmem_relinquish_pair(); }
        else { tmem_alloc(&sh.tmem, p.tmem_cols); tmem_relinquish(); }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    const uint32_t full0 = smem_u32(&sh.full[0]), empty0 = smem_u32(&sh.empty[0]);
    const uint32_t full_mask = PAIR ? PEER_BIT_MASK : 0xFFFFFFFFu;
    auto give_up = [&](int site, int tile) {
        if (!*abort_flag) report_timeout(p.status, site, tile);
        *abort_flag = 1;
    };

    if (warp == 0) {
        if (lane == 0) {
            // ------------------------------------------------------------ loads
            int s = 0, it = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int tile = unit; tile < p.tiles && ok; tile += units, ++it) {
                const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c;
                const int m0 = mt * tile_m + (int)rank * AP_TILE, c0 = ct * p.nt + (int)rank * cols;
                for (int kb = 0; kb < p.kblocks; kb += p.kpb) {
                    if (!mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag)) { give_up(81, tile); ok = false; break; }
                    const int n = min(p.kpb, p.kblocks - kb);
                    const uint32_t fb = (full0 + 8 * s) & full_mask;
                    if (!PAIR || rank == 0) mbar_expect_tx_u32(fb, (PAIR ? 2u : 1u) * (uint32_t)n * (p.a_bytes + p.b_bytes));
                    uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + (uint32_t)p.kpb * p.a_bytes;
                    for (int j = 0; j < n; ++j, a += p.a_bytes, b += p.b_bytes) {
                        const int l = (kb + j) << 6;
                        tma_load_2d_u32<PAIR>(a, &map_z, fb, l, m0, 1u);
                        if (ROWS) for (int g = 0; g < cols >> 6; ++g) tma_load_2d_u32<PAIR>(b + (uint32_t)g * 8192u, &map_w, fb, c0 + 64 * g, l, 1u);
                        else tma_load_2d_u32<PAIR>(b, &map_w, fb, l, c0, 1u);
                    }
                    if (PAIR && rank == 0) mbar_arrive(&sh.full[s]);      // the barrier counts two: in a further block each CTA's builders
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!ok) break;
                const int ib = it & 1;
                if (!mbar_wait(&sh.ifull[ib], (it >> 1) & 1, abort_flag)) { give_up(82, tile); break; }
                const int further = further_stages(p, sh.ext[ib]);
                mbar_arrive(&sh.iempty[ib]);
                // The parity of a barrier tells two neighbouring phases apart and no more: who waits for a stage must know that the use before the
                // last one is over.  The builders know it once this tile's loads are all issued; this thread, for the next tile, where
                // the further blocks are fewer than the stages, and otherwise once they are all built.
                mbar_arrive(&sh.loads[ib]);
                if (further >= p.stages && !mbar_wait(&sh.built[ib], (it >> 1) & 1, abort_flag)) { give_up(91, tile); break; }
                s += further;
                while (s >= p.stages) { s -= p.stages; ph ^= 1; }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            // ------------------------------------------------------------ MMAs
            const uint32_t idesc = make_idesc_bf16(PAIR ? 2 * AP_TILE : AP_TILE, p.nt) | (ROWS ? 1u << 16 : 0u);
            const int tail16 = ((p.L - ((p.kblocks - 1) << 6)) + 15) >> 4;      // steps of 16 in the last block
            constexpr uint32_t b_step = ROWS ? 128u : 2u;
            int s = 0, it = 0;
            uint32_t ph = 0;
            bool ok = true;
            for (int tile = unit; tile < p.tiles && ok; tile += units, ++it) {
                const int ib = it & 1;
                if (!mbar_wait(&sh.tempty[ib], ((it >> 1) & 1) ^ 1, abort_flag)) { give_up(83, tile); break; }
                tc_fence_after();
                const uint32_t d = tmem + (uint32_t)ib * p.acc_cols * (DUAL ? 2u : 1u);
                uint32_t accum = 0;
                for (int kb = 0; kb < p.kblocks; kb += p.kpb) {
                    if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(84, tile); ok = false; break; }
                    tc_fence_after();
                    const int n = min(p.kpb, p.kblocks - kb);
                    uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + (uint32_t)p.kpb * p.a_bytes;
                    for (int j = 0; j < n; ++j, a += p.a_bytes, b += p.b_bytes) {
                        const uint32_t al = sdesc_lo(a), bl = ROWS ? sdesc_rows_lo(b, 8192) : sdesc_lo(b);
                        const int n16 = kb + j == p.kblocks - 1 ? tail16 : 4;
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            umma_bf16_lo<PAIR>(d, al + 2 * k, bl + b_step * k, idesc, accum, k < n16 ? 1u : 0u);
                            accum = 1;
                        }
                    }
                    umma_commit_u32<PAIR>(empty0 + 8 * s);
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!ok) break;
                if (!mbar_wait(&sh.ifull[ib], (it >> 1) & 1, abort_flag)) { give_up(85, tile); break; }
                const int ext = sh.ext[ib];
                const uint32_t de = d + (DUAL ? p.acc_cols : 0u);
                if (DUAL) accum = 0;
                for (int c = 0; c < ext; c += WIDTH * p.kpb) {
                    if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(86, tile); ok = false; break; }
                    tc_fence_after();
                    uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + (uint32_t)p.kpb * p.a_bytes;
                    for (int e = c; e < min(ext, c + WIDTH * p.kpb); e += WIDTH, a += p.a_bytes, b += p.b_bytes) {
                        const int n16 = (TERMS * min(WIDTH, ext - e) + 15) >> 4;
                        const uint32_t al = sdesc_lo(a), bl = ROWS ? sdesc_rows_lo(b, 8192) : sdesc_lo(b);
                        for (int k = 0; k < n16; ++k) {
                            umma_bf16_lo<PAIR>(de, al + 2 * k, bl + b_step * k, idesc, accum, 1u);
                            accum = 1;
                        }
                    }
                    umma_commit_u32<PAIR>(empty0 + 8 * s);
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!ok) break;
                umma_commit_u32<PAIR>(smem_u32(&sh.tfull[ib]));
                mbar_arrive(&sh.iempty[ib]);
            }
        }
        __syncwarp();
    } else if (warp >= 8) {
        // ---------------------------------------------------------------- the rows' adapters, and the further blocks
        const int bt = threadIdx.x - 256;
        int s = 0, it = 0;
        uint32_t ph = 0;
        bool ok = true, waited = false;
        if (p.row_id) { grid_dependency_wait(); waited = true; }               // the rows' adapters, and t, are the kernel's in front
        for (int tile = unit; tile < p.tiles && ok; tile += units, ++it) {
            const int ib = it & 1;
            const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c;
            sh.bits[bt] = 0;
            int id[PAIR ? 2 : 1];
#pragma unroll
            for (int h = 0; h < (PAIR ? 2 : 1); ++h) {
                const int m = mt * tile_m + h * AP_TILE + bt;
                id[h] = !p.row_id ? adapter_of_warp_row(p.rows, m - lane, lane) : m < p.rows.M ? __ldcg(p.row_id + m) : ROW_NONE;
            }
            const bool free_now = mbar_wait(&sh.iempty[ib], ((it >> 1) & 1) ^ 1, abort_flag);
            if (!free_now) give_up(87, tile);
            if (builders_any(!free_now)) break;
#pragma unroll
            for (int h = 0; h < (PAIR ? 2 : 1); ++h) {
                const unsigned same = __match_any_sync(0xffffffffu, id[h]);
                if (id[h] >= 0 && __ffs(same) - 1 == lane) atomicOr(&sh.bits[id[h] >> 5], 1u << (id[h] & 31));
            }
            builders_sync();
            {
                const uint32_t word = sh.bits[bt];
                int n = __popc(word), incl = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += v;
                }
                if (lane == 31) sh.sums[bt >> 5] = incl;
                builders_sync();
                int at = incl - n;
                for (int k = 0; k < (bt >> 5); ++k) at += sh.sums[k];
                sh.before[bt] = at;
                for (uint32_t w = word; w; w &= w - 1) sh.list[ib][at++] = (uint16_t)(bt * 32 + __ffs(w) - 1);
                builders_sync();
            }
            const int own = PAIR ? id[rank] : id[0];
            const int slot = own >= 0 ? sh.before[own >> 5] + __popc(sh.bits[own >> 5] & ((1u << (own & 31)) - 1u)) : own;
            const int used = sh.sums[0] + sh.sums[1] + sh.sums[2] + sh.sums[3];
            const int ext = used * p.Rp;
            sh.slot[ib][bt] = slot;
            if (bt == 0) sh.ext[ib] = ext;
            builders_sync();                            // before the next tile clears the bits
            mbar_arrive(&sh.ifull[ib]);
            s += p.main_stages;
            while (s >= p.stages) { s -= p.stages; ph ^= 1; }

            const int m = mt * tile_m + (int)rank * AP_TILE + bt, c0 = ct * p.nt + (int)rank * cols;
            const float scale = (own >= 0 && p.scale ? __ldg(p.scale + own) : 1.f) * p.factor;
            float* const keep = p.keep && ct == 0 && own != ROW_NONE ? p.keep + (size_t)m * p.R : nullptr;
            if (keep && own == ROW_SHARED)
                for (int r = 0; r < p.R; ++r) keep[r] = 0.f;
            // a thread's pieces of f: of sub-block j its rows row0 + k * step, 16 bytes at cj
            const int cpr = ROWS ? cols >> 3 : 4;                              // 16-byte pieces of a row of a block
            const int cj = bt % cpr, row0 = bt / cpr, step = 128 / cpr;
            const int each = ((ROWS ? WIDTH : cols) + step - 1) / step;        // pieces of a sub-block: kpb * each <= 8
            for (int e0 = 0; e0 < ext; e0 += WIDTH * p.kpb) {
                uint4 fv[8], tv[4][TERMS];
                bool odd = false;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    fv[i] = make_uint4(0, 0, 0, 0);
                    const int j = p.kpb == 1 ? 0 : i / each, row = row0 + (i - j * each) * step;
                    const int eb = e0 + j * WIDTH, w = min(WIDTH, ext - eb);
                    if (j < p.kpb && w > 0 && row < (ROWS ? w : cols) && (ROWS || 8 * cj < w)) {
                        const int e = eb + (ROWS ? row : 8 * cj), d = e / p.Rp, r = e - d * p.Rp;
                        const int a = sh.list[ib][d];
                        if (ROWS) {
                            const int c = c0 + 8 * cj;
                            if (r < p.R && c < p.C) fv[i] = __ldg(reinterpret_cast<const uint4*>(p.f + ((size_t)a * p.R + r) * p.ldf + c));
                        } else if (c0 + row < p.C) {
                            const __nv_bfloat16* src = p.f + ((size_t)a * p.C + c0 + row) * p.R + r;
                            if (p.f_vec) {
                                fv[i] = __ldg(reinterpret_cast<const uint4*>(src));
                            } else {
                                unsigned short h[8];
#pragma unroll
                                for (int q = 0; q < 8; ++q) h[q] = r + q < p.R ? __ldg(reinterpret_cast<const unsigned short*>(src) + q) : (unsigned short)0;
                                fv[i] = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
                            }
                        }
                    }
                }
                if (e0 == 0) {
                    if (!waited) { grid_dependency_wait(); waited = true; }
                    if (p.cache && slot >= 0) {
                        for (int r = 0; r < p.Rp; r += 4) *reinterpret_cast<float4*>(cache + (size_t)bt * p.Rp + r) = __ldcg(reinterpret_cast<const float4*>(p.t + (size_t)m * p.Rp + r));
                        if (keep) for (int r = 0; r < p.R; ++r) keep[r] = cache[(size_t)bt * p.Rp + r];
                    }
                }
                // T of this thread's row in sub-block `eb`
                auto load_t = [&](int eb) {
                    const int w = min(WIDTH, ext - eb);
#pragma unroll
                    for (int j = 0; j < WIDTH / 8; ++j) {
#pragma unroll
                        for (int k = 0; k < TERMS; ++k) tv[j][k] = make_uint4(0, 0, 0, 0);
                        const int r = eb + 8 * j - slot * p.Rp;
                        if (slot >= 0 && r >= 0 && r < p.Rp && 8 * j < w) {
                            float v[8];
                            const float4* src = reinterpret_cast<const float4*>((p.cache ? cache + (size_t)bt * p.Rp : p.t + (size_t)m * p.Rp) + r);
                            const float4 x = p.cache ? src[0] : __ldcg(src), y = p.cache ? src[1] : __ldcg(src + 1);
                            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w; v[4] = y.x; v[5] = y.y; v[6] = y.z; v[7] = y.w;
                            if (keep && !p.cache) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) if (r + i < p.R) keep[r + i] = v[i];
                            }
                            split8<TERMS>(v, scale, tv[j]);
                        }
                    }
                };
                load_t(e0);
#pragma unroll
                for (int i = 0; i < 8; ++i) odd |= finite_only(fv[i]);
                if (odd) {
                    // Both CTAs of a pair drain all columns: each is told.  The number only grows, so that a CTA that runs ahead hides nothing
                    // from one behind; a number ahead of a tile's costs that tile a search for entries it does not have.
                    if (PAIR) {
                        for (uint32_t k = 0; k < 2; ++k)
                            asm volatile("red.relaxed.cluster.shared::cluster.max.s32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&sh.odd[ib]), k)), "r"(it + 1) : "memory");
                    } else {
                        atomicMax(&sh.odd[ib], it + 1);
                    }
                }
                const bool slot_free = __all_sync(0xffffffffu, mbar_wait(&sh.loads[ib], (it >> 1) & 1, abort_flag) &&
                                                                   mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag));
                if (!slot_free) give_up(88, tile);
                if (slot_free) {
                    const uint32_t a0 = ring + (uint32_t)s * p.stage_bytes, b0 = a0 + (uint32_t)p.kpb * p.a_bytes;
                    for (int j = 0; j < p.kpb && e0 + j * WIDTH < ext; ++j) {
                        if (j > 0) load_t(e0 + j * WIDTH);
                        const int w = min(WIDTH, ext - e0 - j * WIDTH), wc = w >> 3;
                        const uint32_t a = a0 + (uint32_t)j * p.a_bytes;
                        if ((uint32_t)bt * 128u < p.a_bytes) {
#pragma unroll
                            for (int i = 0; i < WIDTH / 8; ++i)
                                if (i < wc) {
#pragma unroll
                                    for (int k = 0; k < TERMS; ++k) st_shared16(a + bt * 128 + (((i + k * wc) ^ (bt & 7)) << 4), tv[i][k]);
                                }
                            if (TERMS == 3 && wc == 1) st_shared16(a + bt * 128 + ((3 ^ (bt & 7)) << 4), make_uint4(0, 0, 0, 0));     // 24 columns: two steps of 16
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int j = p.kpb == 1 ? 0 : i / each, row = row0 + (i - j * each) * step;
                        const int w = min(WIDTH, ext - e0 - j * WIDTH), wc = w >> 3;
                        if (j < p.kpb && w > 0 && row < (ROWS ? w : cols) && (ROWS || cj < wc)) {
                            const uint32_t b = b0 + (uint32_t)j * p.b_bytes;
                            if (ROWS) {
                                const uint32_t g = b + (uint32_t)(cj >> 3) * 8192u;
#pragma unroll
                                for (int k = 0; k < TERMS; ++k) st_shared16(g + (row + k * w) * 128 + (((cj & 7) ^ ((row + k * w) & 7)) << 4), fv[i]);
                            } else {
#pragma unroll
                                for (int k = 0; k < TERMS; ++k) st_shared16(b + row * 128 + (((cj + k * wc) ^ (row & 7)) << 4), fv[i]);
                                if (TERMS == 3 && wc == 1) st_shared16(b + row * 128 + ((3 ^ (row & 7)) << 4), make_uint4(0, 0, 0, 0));
                            }
                        }
                    }
                }
                fence_proxy_async_smem();
                if (builders_any(!slot_free)) { ok = false; break; }
                if (bt == 0) {
                    if (PAIR) mbar_arrive_leader(&sh.full[s]);
                    else mbar_arrive(&sh.full[s]);
                }
                if (++s == p.stages) { s = 0; ph ^= 1; }
            }
            if (bt == 0) mbar_arrive(&sh.built[ib]);
        }
        if (!waited) grid_dependency_wait();        // what follows this kernel sees the one in front complete
    } else if (warp >= 4) {
        // ---------------------------------------------------------------- drain
        const int q = warp & 3;
        const uint32_t buf = stage_out + (uint32_t)q * 4096u;
        const bool f32 = p.flags & DR_OUT_F32;
        const unsigned long long off = DUAL ? drop_offset(p.key) : 0ull;
        int it = 0;
        for (int tile = unit; tile < p.tiles; tile += units, ++it) {
            const int ib = it & 1;
            const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c;
            const int n0 = ct * p.nt, n_here = min(p.nt, p.C - n0);
            if (!__all_sync(0xffffffffu, mbar_wait(&sh.ifull[ib], (it >> 1) & 1, abort_flag))) { give_up(89, tile); break; }
            if (p.flags & DR_BIAS)
                for (int c = lane; c < n_here; c += 32) sh.bias[q][c] = __ldg(p.bias + n0 + c);
            const int slot = sh.slot[ib][q * 32 + lane];
            const unsigned valid = __ballot_sync(0xffffffffu, slot != ROW_NONE);
            const int mw = mt * tile_m + (int)rank * AP_TILE + q * 32, m = mw + lane;
            if (!__all_sync(0xffffffffu, mbar_wait(&sh.tfull[ib], (it >> 1) & 1, abort_flag))) { give_up(90, tile); break; }
            tc_fence_after();
            __syncwarp();
            const int ext = sh.ext[ib];
            const bool odd = *(volatile int*)&sh.odd[ib] > it;
            const uint32_t acc = tmem + (uint32_t)ib * p.acc_cols * (DUAL ? 2u : 1u) + ((uint32_t)(q * 32) << 16);
            for (int c = 0; c < n_here; c += 32) {
                uint32_t v[32];
                tmem_ld_x32(acc + c, v);
                tmem_ld_wait();
                if (DUAL && ext) {
                    uint32_t u[32];
                    tmem_ld_x32(acc + p.acc_cols + c, u);
                    tmem_ld_wait();
                    const unsigned long long e = (unsigned long long)m * p.C + n0 + c;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t bits = drop_bits8_at(p.key, off, e + 8 * k);
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (bits >> i & 1) v[8 * k + i] = __float_as_uint(__uint_as_float(v[8 * k + i]) + __uint_as_float(u[8 * k + i]));
                    }
                }
                if (odd && slot >= 0) {
                    const int a = sh.list[ib][slot];
                    const float w = (p.scale ? p.scale[a] : 1.f) * p.factor;
#pragma unroll 1
                    for (int r = 0; r < p.R; ++r) {
                        const float tv = __ldcg(p.t + (size_t)m * p.Rp + r) * w;
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            if (n0 + c + i >= p.C) continue;
                            const float fr = __bfloat162float(ROWS ? p.f[((size_t)a * p.R + r) * p.ldf + n0 + c + i] : p.f[((size_t)a * p.C + n0 + c + i) * p.R + r]);
                            if (!(fabsf(fr) <= 3.4e38f) && (!DUAL || drop_keep_at(p.key, off, (unsigned long long)m * p.C + n0 + c + i)))
                                v[i] = __float_as_uint(fmaf(tv, fr, __uint_as_float(v[i])));
                        }
                    }
                }
                if (p.flags & DR_BIAS) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + sh.bias[q][c + i]);
                }
                if (p.flags & DR_RELU) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(v[i]) < 0.f ? 0u : v[i];      // NaN stays NaN
                }
                // through shared memory, so that a store instruction writes whole rows of 128 bytes: 64 bfloat16 or 32 float32 columns at a time
                if (f32) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        st_shared16(buf + lane * 128 + ((j ^ (lane & 7)) << 4), make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
                } else {
                    const int half = (c >> 5) & 1;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float* x = reinterpret_cast<const float*>(v + 8 * j);
                        st_shared16(buf + lane * 128 + (((4 * half + j) ^ (lane & 7)) << 4),
                                    make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
                    }
                    if (!half && c + 32 < n_here) continue;
                }
                __syncwarp();
                const int first = f32 ? n0 + c : n0 + (c & ~63);
                const int have = min(f32 ? 32 : 64, n0 + n_here - first);
                if (p.out_vec) {
                    const int per = f32 ? 4 : 8, j = lane & 7;
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int row = 4 * k + (lane >> 3);
                        if (!(valid >> row & 1) || j * per >= have) continue;
                        const uint4 x = ld_shared16(buf + row * 128 + ((j ^ (row & 7)) << 4));
                        const size_t at = (size_t)(mw + row) * p.ldo + first + j * per;
                        if (j * per + per <= have) {
                            if (f32) *reinterpret_cast<uint4*>((float*)p.out + at) = x;
                            else *reinterpret_cast<uint4*>((__nv_bfloat16*)p.out + at) = x;
                        } else {
                            const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (i < per && j * per + i < have) {
                                    if (f32) ((uint32_t*)p.out)[at + i] = xs[i & 3];
                                    else ((unsigned short*)p.out)[at + i] = (unsigned short)(xs[i >> 1] >> (16 * (i & 1)));
                                }
                        }
                    }
                } else {
#pragma unroll 1
                    for (int row = 0; row < 32; ++row) {
                        if (!(valid >> row & 1)) continue;
                        for (int i = lane; i < have; i += 32) {
                            const int byte = i * (f32 ? 4 : 2);
                            const uint32_t addr = buf + row * 128 + ((((byte >> 4) ^ (row & 7)) << 4) | (byte & 15));
                            const size_t at = (size_t)(mw + row) * p.ldo + first + i;
                            if (f32) {
                                uint32_t x;
                                asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(addr) : "memory");
                                ((uint32_t*)p.out)[at] = x;
                            } else {
                                unsigned short x;
                                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(addr) : "memory");
                                ((unsigned short*)p.out)[at] = x;
                            }
                        }
                    }
                }
                __syncwarp();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (PAIR) mbar_arrive_leader(&sh.tempty[ib]);
                else mbar_arrive(&sh.tempty[ib]);
                mbar_arrive(&sh.iempty[ib]);
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    if (warp == 1) {
        if (PAIR) tmem_dealloc_pair(tmem, p.tmem_cols);
        else tmem_dealloc(tmem, p.tmem_cols);
    }
}

static int ap_map(CUtensorMap* map, const void* ptr, size_t rows, size_t inner, size_t ld, int box_inner, int box_rows) {
    const cuuint64_t dims[2] = {inner, rows}, strides[1] = {ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows};
    return tmap_tiled(map, 2, ptr, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

template <bool PAIR, bool ROWS, bool DUAL, int TERMS>
static int ap_launch(const CUtensorMap& mz, const CUtensorMap& mw, const ApParams& p, bool overlap, size_t smem, cudaStream_t s) {
    static PerDeviceFlag ready;
    auto* k = adapter_product_kernel<PAIR, ROWS, DUAL, TERMS>;
    if (!ready.get()) {
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 8192 - 1024) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
        ready.set();
    }
    cudaLaunchConfig_t cfg = {};
    const int units = PAIR ? num_sms() / 2 : num_sms();
    cfg.gridDim = dim3((unsigned)(std::min(p.tiles, units) * (PAIR ? 2 : 1)));
    cfg.blockDim = dim3(AP_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (PAIR) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = 2; attr[n].val.clusterDim.y = 1; attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (overlap) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cfg.attrs = attr;
    cfg.numAttrs = n;
    if (cudaLaunchKernelEx(&cfg, k, mz, mw, p) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
    count_launch();
    return DR_OK;
}

int adapter_product_run(const ProductArgs& a, bool overlap, cudaStream_t s) {
    ApParams p = {};
    p.rows = a.rows;
    p.L = a.L; p.C = a.C; p.R = a.R; p.Rp = a.Rp;
    p.t = a.t; p.scale = a.scale; p.bias = a.bias; p.f = a.f; p.ldf = a.ldf; p.factor = a.factor; p.keep = a.keep;
    p.f_vec = !a.transposed && (a.R & 7) == 0;
    p.flags = a.flags; p.out = a.out; p.ldo = a.ldo; p.key = a.key;
    const size_t size = (a.flags & DR_OUT_F32) ? 4 : 2;
    p.out_vec = aligned16(a.out) && (a.ldo * size) % 16 == 0;
    p.status = dev_status_ptr();
    const bool dual = a.key.thr != 0;
    const int M = a.rows.M, sms = num_sms();
    const long long rows128 = (M + 127) / 128;
    const int gran = a.transposed ? 64 : 16;
    // Tile: as wide as leaves every SM one, by pairs where the pairs have enough tiles
    const int most = dual ? 128 : 256;
    bool pair = false;
    int nt = std::min(most, (a.C + gran - 1) / gran * gran);
    if (rows128 * ((a.C + nt - 1) / nt) < sms) {
        const long long want = std::max(1ll, sms / rows128);         // column blocks that give every SM a tile
        nt = (int)((a.C + want - 1) / want);
        nt = std::min(most, std::max(gran, (nt + gran - 1) / gran * gran));
    } else if (M > 128 && a.C >= 128) {
        const int pn = a.C > 128 ? most : 128;
        const long long pairs = ((rows128 + 1) / 2) * ((a.C + pn - 1) / pn);
        if (pairs >= sms / 2) { pair = true; nt = pn; }
    }
    p.nt = nt;
    p.tiles_c = (a.C + nt - 1) / nt;
    const long long tiles = (pair ? (rows128 + 1) / 2 : rows128) * p.tiles_c;
    if (tiles > 0x7fffffffll) return DR_ERR_UNSUPPORTED;
    p.tiles = (int)tiles;
    const int cols = pair ? nt / 2 : nt;
    const int a_rows = std::min(128, (M + 7) / 8 * 8);
    p.a_bytes = (uint32_t)a_rows * 128u;
    p.b_bytes = (uint32_t)cols * 128u;
    p.kblocks = (a.L + 63) / 64;
    const uint32_t block = p.a_bytes + p.b_bytes;
    p.kpb = block <= 8192 ? 4 : block <= 16384 ? 2 : 1;
    p.kpb = std::min(p.kpb, p.kblocks);
    p.terms = (a.flags & DR_OUT_F32) ? 3 : 2;
    p.width = p.terms == 2 ? 32 : 16;
    p.row_id = M > AP_TILE ? a.row_id : nullptr;
    p.cache = p.kpb > 1 ? (M * a.Rp * 4 + 1023) / 1024 * 1024 : 0;
    if (p.cache > AP_CACHE) { p.cache = 0; p.kpb = 1; }
    p.main_stages = (p.kblocks + p.kpb - 1) / p.kpb;
    p.stage_bytes = (uint32_t)p.kpb * block;
    const uint32_t slack = p.a_bytes < 16384u ? 16384u - p.a_bytes : 0u;      // the MMA reads 128 rows from the last stage on
    p.stages = (int)std::min<uint32_t>(AP_MAX_STAGES, (AP_SMEM - p.cache - slack) / p.stage_bytes);
    p.acc_cols = 32;
    while ((int)p.acc_cols < nt) p.acc_cols *= 2;
    p.tmem_cols = p.acc_cols * (dual ? 4 : 2);
    const size_t smem = 1024 + (size_t)p.stages * p.stage_bytes + slack + 4 * 4096 + p.cache;
    alignas(64) CUtensorMap mz, mw;
    int rc = ap_map(&mz, a.z, M, a.L, a.ldz, 64, a_rows);
    if (rc != DR_OK) return rc;
    rc = a.transposed ? ap_map(&mw, a.w, a.L, a.C, a.ldw, 64, 64) : ap_map(&mw, a.w, a.C, a.L, a.ldw, 64, cols);
    if (rc != DR_OK) return rc;
    const bool f32 = p.terms == 3;
    if (a.transposed) {
        if (pair) return dual ? ap_launch<true, true, true, 2>(mz, mw, p, overlap, smem, s) : ap_launch<true, true, false, 2>(mz, mw, p, overlap, smem, s);
        return dual ? ap_launch<false, true, true, 2>(mz, mw, p, overlap, smem, s) : ap_launch<false, true, false, 2>(mz, mw, p, overlap, smem, s);
    }
    if (pair) return f32 ? ap_launch<true, false, false, 3>(mz, mw, p, overlap, smem, s) : ap_launch<true, false, false, 2>(mz, mw, p, overlap, smem, s);
    return f32 ? ap_launch<false, false, false, 3>(mz, mw, p, overlap, smem, s) : ap_launch<false, false, false, 2>(mz, mw, p, overlap, smem, s);
}

}  // namespace dr
