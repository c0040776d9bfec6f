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
// 16 warps: 0 loads (TMA), 1 (and 2) issue MMAs, 4-11 drain, 12-15 find the rows' adapters and build the further blocks in the ring's
// stages.  A CTA's first tile takes them behind its blocks of l, so that w streams in while t is still being made; later tiles take them in front, so
// that they are built while the tile before is multiplied.
#include <algorithm>

#include "adapter.cuh"
#include "conv_common.cuh"
#include "umma_ptx.cuh"

namespace dr {
using namespace ptx;

constexpr int AP_THREADS = 512;
constexpr int AP_MAX_STAGES = 16;
constexpr int AP_SMEM = 184 * 1024;     // the ring's; with 32 KB of the drain's and the barriers' all of an SM's
constexpr int AP_SMEM_MOST = 217 * 1024;
constexpr int AP_TILE = 128;
constexpr int AP_CACHE = 32 * 1024;     // T of a tile of few rows

struct ApParams {
    AdRows rows;
    int L, C, R, Rp;
    uint32_t rp_magic;          // 2^32 / Rp, rounded up: columns / Rp by a multiplication
    int nt;                     // columns of a tile
    int tiles_c, tiles;
    int kblocks, main_stages, stages;
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
    alignas(16) float bias[2][512];
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

// What one kernel is compiled for.  KPB: blocks of 64 l to a stage.  PAIR: tiles of 256 rows by two CTAs.  WIDE (pairs): two accumulators of 256
// columns share the rows' blocks, each with an issuing warp of its own.  ROWS: w and f have the contraction index as their rows.  DUAL: an
// accumulator of its own for the adapters.  TERMS: bfloat16 values to a T.
template <int KPB_, bool PAIR_, bool WIDE_, bool ROWS_, bool DUAL_, int TERMS_>
struct ApKind {
    static constexpr int KPB = KPB_, TERMS = TERMS_;
    static constexpr bool PAIR = PAIR_, WIDE = WIDE_, ROWS = ROWS_, DUAL = DUAL_;
    static constexpr int WIDTH = TERMS == 2 ? 32 : 16;         // columns of T in a further block of 64
    static constexpr int STAGE_WIDTH = WIDTH * KPB;
    static constexpr int EACH = 8 / KPB;                        // 16-byte pieces of a block's f that a thread brings
};
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <class Kind>
__global__ void __launch_bounds__(AP_THREADS, 1)
adapter_product_kernel(const __grid_constant__ CUtensorMap map_z, const __grid_constant__ CUtensorMap map_w, const ApParams p) {
    constexpr bool PAIR = Kind::PAIR, WIDE = Kind::WIDE, ROWS = Kind::ROWS, DUAL = Kind::DUAL;
    constexpr int KPB = Kind::KPB, TERMS = Kind::TERMS, WIDTH = Kind::WIDTH;
    extern __shared__ uint8_t ap_raw[];
    __shared__ ApShared sh;
    const uint32_t ring = (smem_u32(ap_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = PAIR ? cluster_ctarank() : 0u;
    const int unit = PAIR ? (int)blockIdx.x >> 1 : (int)blockIdx.x, units = PAIR ? (int)gridDim.x >> 1 : (int)gridDim.x;
    constexpr int tile_m = PAIR ? 2 * AP_TILE : AP_TILE;
    const int cols = PAIR ? p.nt >> 1 : p.nt;                  // columns of w that this CTA loads
    // column of the output that place i of them is: a wide tile's halves are 256 columns apart, 128 of each in either CTA
    auto column = [&](int i) { return WIDE ? (i >> 7) * 256 + (int)rank * 128 + (i & 127) : (int)rank * cols + i; };
    volatile int* abort_flag = &sh.abort;
    // after the ring, 4 KB for each draining warp, and T of a tile of few rows
    const uint32_t stage_out = ring + (uint32_t)p.stages * p.stage_bytes + (p.a_bytes < 16384u ? 16384u - p.a_bytes : 0u);
    float* const cache = reinterpret_cast<float*>(ap_raw + (stage_out + 8 * 4096u - smem_u32(ap_raw)));
    auto further_stages = [](int ext) { return (ext + Kind::STAGE_WIDTH - 1) / Kind::STAGE_WIDTH; };

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { mbar_init(&sh.full[i], PAIR ? 2 : 1); mbar_init(&sh.empty[i], WIDE ? 2 : 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.tfull[i], 1);
            mbar_init(&sh.tempty[i], PAIR ? 16 : 8);
            mbar_init(&sh.loads[i], 1);
            mbar_init(&sh.built[i], 1);
            mbar_init(&sh.ifull[i], 128);
            mbar_init(&sh.iempty[i], 9 + (rank == 0 ? (WIDE ? 2 : 1) : 0));
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
            int s = 0, it = 0, gap = 0;
            uint32_t ph = 0;
            bool ok = true;
            // Passes over the further blocks of a tile.  The parity of a barrier tells two neighbouring phases apart and no more: who waits for a stage
            // must know that the use before the last one is over.  The builders know it once the loads in front of theirs are all
            // issued (sh.loads); this thread where the further blocks since its last load are fewer than the stages, and otherwise once they are
            // built.
            auto pass = [&](int tile) {
                const int ib = it & 1;
                if (!mbar_wait(&sh.ifull[ib], (it >> 1) & 1, abort_flag)) { give_up(82, tile); return false; }
                const int further = further_stages(sh.ext[ib]);
                mbar_arrive(&sh.iempty[ib]);
                gap += further;
                if (it > 0 && gap >= p.stages && !mbar_wait(&sh.built[ib], (it >> 1) & 1, abort_flag)) { give_up(91, tile); return false; }
                s += further;
                while (s >= p.stages) { s -= p.stages; ph ^= 1; }
                return true;
            };
            for (int tile = unit; tile < p.tiles && ok; tile += units, ++it) {
                const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c;
                const int m0 = mt * tile_m + (int)rank * AP_TILE, c0 = ct * p.nt;
                if (it > 0 && !pass(tile)) break;
                for (int kb = 0; kb < p.kblocks; kb += KPB) {
                    if (!mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag)) { give_up(81, tile); ok = false; break; }
                    const int n = min(KPB, p.kblocks - kb);
                    const uint32_t fb = (full0 + 8 * s) & full_mask;
                    if (!PAIR || rank == 0) mbar_expect_tx_u32(fb, (PAIR ? 2u : 1u) * (uint32_t)n * (p.a_bytes + p.b_bytes));
                    uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + (uint32_t)KPB * p.a_bytes;
#pragma unroll
                    for (int j = 0; j < KPB; ++j, a += p.a_bytes, b += p.b_bytes) {
                        if (j >= n) break;
                        const int l = (kb + j) << 6;
                        tma_load_2d_u32<PAIR>(a, &map_z, fb, l, m0, 1u);
                        if (ROWS) {
                            for (int g = 0; g < cols >> 6; ++g) tma_load_2d_u32<PAIR>(b + (uint32_t)g * 8192u, &map_w, fb, c0 + column(64 * g), l, 1u);
                        } else {
                            tma_load_2d_u32<PAIR>(b, &map_w, fb, l, c0 + column(0), 1u);
                            if (WIDE) tma_load_2d_u32<PAIR>(b + 16384u, &map_w, fb, l, c0 + column(128), 1u);
                        }
                    }
                    if (PAIR && rank == 0) mbar_arrive(&sh.full[s]);      // the barrier counts two: in a further block each CTA's builders
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!ok) break;
                gap = 0;
                mbar_arrive(&sh.loads[it & 1]);
                if (it == 0 && !pass(tile)) break;
            }
        }
        __syncwarp();
    } else if (warp == 1 || (WIDE && warp == 2)) {
        if (lane == 0 && rank == 0) {
            // ------------------------------------------------------------ MMAs
            const int half = WIDE ? warp - 1 : 0;
            const uint32_t idesc = make_idesc_bf16(PAIR ? 2 * AP_TILE : AP_TILE, WIDE ? 256 : p.nt) | (ROWS ? 1u << 16 : 0u);
            const int tail16 = ((p.L - ((p.kblocks - 1) << 6)) + 15) >> 4;      // steps of 16 in the last block
            constexpr uint32_t b_step = ROWS ? 128u : 2u;
            int s = 0, it = 0;
            uint32_t ph = 0, accum = 0, d = 0;
            auto further = [&](int tile) {
                const int ib = it & 1;
                if (!mbar_wait(&sh.ifull[ib], (it >> 1) & 1, abort_flag)) { give_up(85, tile); return false; }
                const int ext = sh.ext[ib];
                mbar_arrive(&sh.iempty[ib]);
                const uint32_t de = d + (DUAL ? p.acc_cols : 0u);
                uint32_t acc = DUAL ? 0u : accum;
                for (int c = 0; c < ext; c += Kind::STAGE_WIDTH) {
                    if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(86, tile); return false; }
                    tc_fence_after();
                    uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + (uint32_t)KPB * p.a_bytes + (uint32_t)half * 16384u;
                    for (int e = c; e < min(ext, c + Kind::STAGE_WIDTH); e += WIDTH, a += p.a_bytes, b += p.b_bytes) {
                        const int n16 = (TERMS * min(WIDTH, ext - e) + 15) >> 4;
                        const uint32_t al = sdesc_lo(a), bl = ROWS ? sdesc_rows_lo(b, 8192) : sdesc_lo(b);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            umma_bf16_lo<PAIR>(de, al + 2 * k, bl + b_step * k, idesc, acc, k < n16 ? 1u : 0u);
                            acc = 1;
                        }
                    }
                    umma_commit_u32<PAIR>(empty0 + 8 * s);
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!DUAL) accum = acc;
                return true;
            };
            for (int tile = unit; tile < p.tiles; tile += units, ++it) {
                const int ab = WIDE ? half : it & 1, use = WIDE ? it : it >> 1;        // accumulator and how often it was used
                if (!mbar_wait(&sh.tempty[ab], (use & 1) ^ 1, abort_flag)) { give_up(83, tile); break; }
                tc_fence_after();
                d = tmem + (uint32_t)ab * p.acc_cols * (DUAL ? 2u : 1u);
                accum = 0;
                if (it > 0 && !further(tile)) break;
                bool ok = true;
                for (int kb = 0; kb < p.kblocks; kb += KPB) {
                    if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(84, tile); ok = false; break; }
                    tc_fence_after();
                    const int n = min(KPB, p.kblocks - kb);
                    uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + (uint32_t)KPB * p.a_bytes + (uint32_t)half * 16384u;
#pragma unroll
                    for (int j = 0; j < KPB; ++j, a += p.a_bytes, b += p.b_bytes) {
                        if (j >= n) break;
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
                if (!ok || (it == 0 && !further(tile))) break;
                umma_commit_u32<PAIR>(smem_u32(&sh.tfull[ab]));
            }
        }
        __syncwarp();
    } else if (warp >= 12) {
        // ---------------------------------------------------------------- the rows' adapters, and the further blocks
        const int bt = threadIdx.x - 384;
        int s = 0, it = 0;
        uint32_t ph = 0;
        bool ok = true, waited = false;
        auto advance = [&](int n) {
            s += n;
            while (s >= p.stages) { s -= p.stages; ph ^= 1; }
        };
        if (p.row_id) { grid_dependency_wait(); waited = true; }               // the rows' adapters, and t, are the kernel's in front
        // a thread's pieces of f: of a block its rows row0 + k * step, 16 bytes at cj
        const int cpr = ROWS ? cols >> 3 : 4;                                  // 16-byte pieces of a row of a block
        const int cj = bt % cpr, row0 = bt / cpr, step = 128 / cpr;
        for (int tile = unit; tile < p.tiles && ok; tile += units, ++it) {
            const int ib = it & 1;
            const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c, c0 = ct * p.nt;
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
            if (p.flags & DR_BIAS)
                for (int c = bt; c < p.nt; c += 128) sh.bias[ib][c] = c0 + c < p.C ? __ldg(p.bias + c0 + c) : 0.f;
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
            const int ext = (sh.sums[0] + sh.sums[1] + sh.sums[2] + sh.sums[3]) * p.Rp;
            sh.slot[ib][bt] = slot;
            if (bt == 0) sh.ext[ib] = ext;
            builders_sync();                            // before the next tile clears the bits
            mbar_arrive(&sh.ifull[ib]);
            if (it == 0) advance(p.main_stages);

            const int m = mt * tile_m + (int)rank * AP_TILE + bt;
            const float scale = (own >= 0 && p.scale ? __ldg(p.scale + own) : 1.f) * p.factor;
            float* const keep = p.keep && ct == 0 && own != ROW_NONE ? p.keep + (size_t)m * p.R : nullptr;
            if (keep && own == ROW_SHARED)
                for (int r = 0; r < p.R; ++r) keep[r] = 0.f;
            const float* const trow = KPB > 1 ? cache + (size_t)bt * p.Rp : p.t + (size_t)m * p.Rp;
            for (int e0 = 0; e0 < ext; e0 += Kind::STAGE_WIDTH) {
                uint4 fv[8], tv[WIDTH / 8][TERMS];
#pragma unroll
                for (int j = 0; j < KPB; ++j) {
                    const int eb = e0 + j * WIDTH, w = min(WIDTH, ext - eb);
                    const int ef = eb + 8 * cj, df = (int)__umulhi((uint32_t)ef, p.rp_magic), rf = ef - df * p.Rp;
                    const int af = !ROWS && 8 * cj < w ? sh.list[ib][df] : 0;
#pragma unroll
                    for (int i = 0; i < Kind::EACH; ++i) {
                        uint4& v = fv[j * Kind::EACH + i];
                        v = make_uint4(0, 0, 0, 0);
                        const int row = row0 + i * step;
                        if (ROWS) {
                            const int c = c0 + column(8 * cj);
                            if (row < w && c < p.C) {
                                const int e = eb + row, dd = (int)__umulhi((uint32_t)e, p.rp_magic), r = e - dd * p.Rp;
                                if (r < p.R) v = __ldg(reinterpret_cast<const uint4*>(p.f + ((size_t)sh.list[ib][dd] * p.R + r) * p.ldf + c));
                            }
                        } else {
                            const int c = c0 + column(row);
                            if (8 * cj < w && row < cols && c < p.C) {
                                const __nv_bfloat16* src = p.f + ((size_t)af * p.C + c) * p.R + rf;
                                if (p.f_vec) {
                                    v = __ldg(reinterpret_cast<const uint4*>(src));
                                } else {
                                    unsigned short h[8];
#pragma unroll
                                    for (int q = 0; q < 8; ++q) h[q] = rf + q < p.R ? __ldg(reinterpret_cast<const unsigned short*>(src) + q) : (unsigned short)0;
                                    v = make_uint4(h[0] | (uint32_t)h[1] << 16, h[2] | (uint32_t)h[3] << 16, h[4] | (uint32_t)h[5] << 16, h[6] | (uint32_t)h[7] << 16);
                                }
                            }
                        }
                    }
                }
                if (!waited) { grid_dependency_wait(); waited = true; }
                if (KPB > 1 && e0 == 0 && slot >= 0) {
                    for (int r = 0; r < p.Rp; r += 4) *reinterpret_cast<float4*>(cache + (size_t)bt * p.Rp + r) = __ldcg(reinterpret_cast<const float4*>(p.t + (size_t)m * p.Rp + r));
                    if (keep) for (int r = 0; r < p.R; ++r) keep[r] = cache[(size_t)bt * p.Rp + r];
                }
                // T of this thread's row in the block `eb`
                auto load_t = [&](int eb) {
                    const int w = min(WIDTH, ext - eb);
#pragma unroll
                    for (int j = 0; j < WIDTH / 8; ++j) {
#pragma unroll
                        for (int k = 0; k < TERMS; ++k) tv[j][k] = make_uint4(0, 0, 0, 0);
                        const int r = eb + 8 * j - slot * p.Rp;
                        if (slot >= 0 && r >= 0 && r < p.Rp && 8 * j < w) {
                            const float4* src = reinterpret_cast<const float4*>(trow + r);
                            const float4 x = KPB > 1 ? src[0] : __ldcg(src), y = KPB > 1 ? src[1] : __ldcg(src + 1);
                            const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                            if (KPB == 1 && keep) {
#pragma unroll
                                for (int i = 0; i < 8; ++i) if (r + i < p.R) keep[r + i] = v[i];
                            }
                            split8<TERMS>(v, scale, tv[j]);
                        }
                    }
                };
                load_t(e0);
                bool odd = false;
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
                const int before = it == 0 ? 0 : it - 1;        // the tile whose loads lie in front of this block
                const bool slot_free = __all_sync(0xffffffffu, mbar_wait(&sh.loads[before & 1], (before >> 1) & 1, abort_flag) &&
                                                                   mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag));
                if (!slot_free) give_up(88, tile);
                if (slot_free) {
                    uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + (uint32_t)KPB * p.a_bytes;
#pragma unroll
                    for (int j = 0; j < KPB; ++j, a += p.a_bytes, b += p.b_bytes) {
                        const int eb = e0 + j * WIDTH, w = min(WIDTH, ext - eb), wc = w >> 3;
                        if (w <= 0) break;
                        if (j > 0) load_t(eb);
                        if ((uint32_t)bt * 128u < p.a_bytes) {
                            const uint32_t at = a + bt * 128, x = (uint32_t)(bt & 7);
#pragma unroll
                            for (int i = 0; i < WIDTH / 8; ++i)
                                if (i < wc) {
#pragma unroll
                                    for (int k = 0; k < TERMS; ++k) st_shared16(at + (((uint32_t)(i + k * wc) ^ x) << 4), tv[i][k]);
                                }
                            if (TERMS == 3 && wc == 1) st_shared16(at + ((3u ^ x) << 4), make_uint4(0, 0, 0, 0));     // 24 columns: two steps of 16
                        }
#pragma unroll
                        for (int i = 0; i < Kind::EACH; ++i) {
                            const uint4& v = fv[j * Kind::EACH + i];
                            const int row = row0 + i * step;
                            if (ROWS) {
                                if (row < w) {
                                    const uint32_t g = b + (uint32_t)(cj >> 3) * 8192u;
#pragma unroll
                                    for (int k = 0; k < TERMS; ++k) st_shared16(g + (row + k * w) * 128 + (((cj & 7) ^ ((row + k * w) & 7)) << 4), v);
                                }
                            } else if (row < cols && cj < wc) {
                                const uint32_t at = b + row * 128, x = (uint32_t)(row & 7);
#pragma unroll
                                for (int k = 0; k < TERMS; ++k) st_shared16(at + (((uint32_t)(cj + k * wc) ^ x) << 4), v);
                                if (TERMS == 3 && wc == 1) st_shared16(at + ((3u ^ x) << 4), make_uint4(0, 0, 0, 0));
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
                advance(1);
            }
            if (bt == 0) mbar_arrive(&sh.built[ib]);
            if (it > 0) advance(p.main_stages);
        }
        if (!waited) grid_dependency_wait();        // what follows this kernel sees the one in front complete
    } else if (warp >= 4) {
        // ---------------------------------------------------------------- drain: two warps to a quarter of the rows, every other 128 bytes of columns each
        const int q = warp & 3, side = (warp - 4) >> 2;
        const uint32_t buf = stage_out + (uint32_t)(warp - 4) * 4096u;
        const uint32_t put = buf + lane * 128, px = (uint32_t)(lane & 7), get = buf + (lane >> 3) * 128;
        const bool f32 = TERMS == 3;
        constexpr int CHUNK = TERMS == 3 ? 32 : 64;                            // columns of 128 bytes
        const float low = (p.flags & DR_RELU) ? 0.f : -INFINITY;
        const uint32_t low2 = (p.flags & DR_RELU) ? 0u : 0xFF80FF80u;
        const size_t size = f32 ? 4 : 2;
        const unsigned long long off = DUAL ? drop_offset(p.key) : 0ull;
        int it = 0;
        bool ok = true;
        for (int tile = unit; tile < p.tiles && ok; tile += units, ++it) {
            const int ib = it & 1;
            const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c;
            const int n0 = ct * p.nt, n_here = min(p.nt, p.C - n0);
            if (!__all_sync(0xffffffffu, mbar_wait(&sh.ifull[ib], (it >> 1) & 1, abort_flag))) { give_up(89, tile); break; }
            const int slot = sh.slot[ib][q * 32 + lane];
            const unsigned valid = __ballot_sync(0xffffffffu, slot != ROW_NONE);
            const int mw = mt * tile_m + (int)rank * AP_TILE + q * 32, m = mw + lane;
            const int ext = sh.ext[ib];
            char* const rowp = (char*)p.out + ((size_t)(mw + (lane >> 3)) * p.ldo + n0) * size + (lane & 7) * 16;
            const size_t row4 = 4 * p.ldo * size;
            const uint32_t quarter = (uint32_t)(q * 32) << 16;
#pragma unroll 1
            for (int part = 0; part < (WIDE ? 2 : 1); ++part) {
                const int ab = WIDE ? part : ib, use = WIDE ? it : it >> 1;
                if (!__all_sync(0xffffffffu, mbar_wait(&sh.tfull[ab], use & 1, abort_flag))) { give_up(90, tile); ok = false; break; }
                tc_fence_after();
                const bool odd = *(volatile int*)&sh.odd[ib] > it;
                const uint32_t acc = tmem + (uint32_t)ab * p.acc_cols * (DUAL ? 2u : 1u) + quarter;
                const int c_end = WIDE ? min(256, n_here - 256 * part) : n_here, cb = WIDE ? 256 * part : 0;
#pragma unroll 1
                for (int c = side * CHUNK; c < c_end; c += 2 * CHUNK) {
                    uint32_t v[CHUNK];
#pragma unroll
                    for (int h = 0; h < CHUNK; h += 32) tmem_ld_x32(acc + c + h, v + h);
                    tmem_ld_wait();
                    if (DUAL && ext) {
#pragma unroll
                        for (int h = 0; h < CHUNK; h += 8) {
                            uint32_t u[8];
                            tmem_ld_x8(acc + p.acc_cols + c + h, u);
                            const uint32_t bits = drop_bits8_at(p.key, off, (unsigned long long)m * p.C + n0 + c + h);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (bits >> i & 1) v[h + i] = __float_as_uint(__uint_as_float(v[h + i]) + __uint_as_float(u[i]));
                        }
                    }
                    if (odd && slot >= 0) {
                        const int a = sh.list[ib][slot];
                        const float w = (p.scale ? p.scale[a] : 1.f) * p.factor;
#pragma unroll 1
                        for (int r = 0; r < p.R; ++r) {
                            const float tv = __ldcg(p.t + (size_t)m * p.Rp + r) * w;
#pragma unroll
                            for (int i = 0; i < CHUNK; ++i) {
                                const int col = n0 + cb + c + i;
                                if (col >= p.C) continue;
                                const float fr = __bfloat162float(ROWS ? p.f[((size_t)a * p.R + r) * p.ldf + col] : p.f[((size_t)a * p.C + col) * p.R + r]);
                                if (!(fabsf(fr) <= 3.4e38f) && (!DUAL || drop_keep_at(p.key, off, (unsigned long long)m * p.C + col)))
                                    v[i] = __float_as_uint(fmaf(tv, fr, __uint_as_float(v[i])));
                            }
                        }
                    }
                    if (p.flags & DR_BIAS) {
                        const float4* bias = reinterpret_cast<const float4*>(&sh.bias[ib][cb + c]);
#pragma unroll
                        for (int i = 0; i < CHUNK / 4; ++i) {
                            const float4 x = bias[i];
                            v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + x.x);
                            v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + x.y);
                            v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + x.z);
                            v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + x.w);
                        }
                    }
                    // through shared memory, so that a store instruction writes whole rows of 128 bytes
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        uint4 x;
                        if (f32) {
                            float y[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[i] = max_nan(__uint_as_float(v[(4 * j + i) % CHUNK]), low);
                            x = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
                        } else {
                            const float* y = reinterpret_cast<const float*>(v + (8 * j) % CHUNK);
                            x = make_uint4(max_nan_bf16x2(pack_bf16(y[0], y[1]), low2), max_nan_bf16x2(pack_bf16(y[2], y[3]), low2),
                                           max_nan_bf16x2(pack_bf16(y[4], y[5]), low2), max_nan_bf16x2(pack_bf16(y[6], y[7]), low2));
                        }
                        st_shared16(put + (((uint32_t)j ^ px) << 4), x);
                    }
                    __syncwarp();
                    const int have = min(CHUNK, c_end - c);
                    if (p.out_vec) {
                        const int per = f32 ? 4 : 8, j = lane & 7;
                        char* to = rowp + (size_t)(cb + c) * size;
                        const bool whole = j * per + per <= have;
#pragma unroll
                        for (int k = 0; k < 8; ++k, to += row4) {
                            const int row = 4 * k + (lane >> 3);
                            if (!(valid >> row & 1) || j * per >= have) continue;
                            const uint4 x = ld_shared16(get + 512 * k + (((uint32_t)j ^ (uint32_t)(row & 7)) << 4));
                            if (whole) {
                                *reinterpret_cast<uint4*>(to) = x;
                            } else {
                                const uint32_t xs[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                                for (int i = 0; i < 8; ++i)
                                    if (i < per && j * per + i < have) {
                                        if (f32) ((uint32_t*)to)[i] = xs[i & 3];
                                        else ((unsigned short*)to)[i] = (unsigned short)(xs[i >> 1] >> (16 * (i & 1)));
                                    }
                            }
                        }
                    } else {
#pragma unroll 4
                        for (int row = 0; row < 32; ++row) {
                            if (!(valid >> row & 1)) continue;
#pragma unroll
                            for (int i = lane; i < CHUNK; i += 32) {
                                if (i >= have) continue;
                                const int byte = i * (f32 ? 4 : 2);
                                const uint32_t addr = buf + row * 128 + ((((byte >> 4) ^ (row & 7)) << 4) | (byte & 15));
                                const size_t at = (size_t)(mw + row) * p.ldo + n0 + cb + c + i;
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
                    if (PAIR) mbar_arrive_leader(&sh.tempty[ab]);
                    else mbar_arrive(&sh.tempty[ab]);
                }
            }
            if (lane == 0) mbar_arrive(&sh.iempty[ib]);
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

template <class Kind>
static int ap_launch(const CUtensorMap& mz, const CUtensorMap& mw, const ApParams& p, bool overlap, size_t smem, cudaStream_t s) {
    static PerDeviceFlag ready;
    auto* k = adapter_product_kernel<Kind>;
    if (!ready.get()) {
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, AP_SMEM_MOST) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
        ready.set();
    }
    cudaLaunchConfig_t cfg = {};
    const int units = Kind::PAIR ? num_sms() / 2 : num_sms();
    cfg.gridDim = dim3((unsigned)(std::min(p.tiles, units) * (Kind::PAIR ? 2 : 1)));
    cfg.blockDim = dim3(AP_THREADS);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (Kind::PAIR) {
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
    p.rp_magic = (uint32_t)((0x100000000ull + a.Rp - 1) / a.Rp);
    p.t = a.t; p.scale = a.scale; p.bias = a.bias; p.f = a.f; p.ldf = a.ldf; p.factor = a.factor; p.keep = a.keep;
    p.f_vec = !a.transposed && (a.R & 7) == 0;
    p.flags = a.flags; p.out = a.out; p.ldo = a.ldo; p.key = a.key;
    const size_t size = (a.flags & DR_OUT_F32) ? 4 : 2;
    p.out_vec = aligned16(a.out) && (a.ldo * size) % 16 == 0;
    p.status = dev_status_ptr();
    const bool dual = a.key.thr != 0, f32 = a.flags & DR_OUT_F32;
    const int M = a.rows.M, sms = num_sms();
    const long long rows128 = (M + 127) / 128;
    const int gran = a.transposed ? 64 : 16;
    // Tile: as wide as leaves every SM one, by pairs where the pairs have enough tiles
    const int most = dual ? 128 : 256;
    bool pair = false, wide = false;
    int nt = std::min(most, (a.C + gran - 1) / gran * gran);
    if (rows128 * ((a.C + nt - 1) / nt) < sms) {
        const long long want = std::max(1ll, sms / rows128);         // column blocks that give every SM a tile
        nt = (int)((a.C + want - 1) / want);
        nt = std::min(most, std::max(gran, (nt + gran - 1) / gran * gran));
    } else if (M > 128 && a.C >= 128) {
        const int pn = a.C > 128 ? most : 128;
        const long long pairs = ((rows128 + 1) / 2) * ((a.C + pn - 1) / pn);
        if (pairs >= sms / 2) { pair = true; nt = pn; }
        // Out of L2 a pair's block of 256 x 256 takes 64 KB for 512 cycles of MMAs, more than the 12 TB/s that all SMs get; 256 x 512 takes 96 KB
        // for 1024, but its accumulators fill the tensor memory, so a tile's drain is only half hidden: long l
        if (pair && !dual && a.L >= 1024 && a.C >= 512 && ((rows128 + 1) / 2) * ((a.C + 511) / 512) >= sms / 2) { wide = true; nt = 512; }
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
    int kpb = block <= 8192 ? 4 : block <= 16384 ? 2 : 1;
    if (kpb > 1) {
        p.cache = (M * a.Rp * 4 + 1023) / 1024 * 1024;
        if (p.cache > AP_CACHE) { p.cache = 0; kpb = 1; }
    }
    p.row_id = M > AP_TILE ? a.row_id : nullptr;
    p.main_stages = (p.kblocks + kpb - 1) / kpb;
    p.stage_bytes = (uint32_t)kpb * block;
    const uint32_t slack = p.a_bytes < 16384u ? 16384u - p.a_bytes : 0u;      // the MMA reads 128 rows from the last stage on
    p.stages = (int)std::min<uint32_t>(AP_MAX_STAGES, (AP_SMEM - p.cache - slack) / p.stage_bytes);
    p.acc_cols = 32;
    while ((int)p.acc_cols < (wide ? 256 : nt)) p.acc_cols *= 2;
    p.tmem_cols = p.acc_cols * (dual ? 4 : 2);
    const size_t smem = 1024 + (size_t)p.stages * p.stage_bytes + slack + 8 * 4096 + p.cache;
    alignas(64) CUtensorMap mz, mw;
    int rc = ap_map(&mz, a.z, M, a.L, a.ldz, 64, a_rows);
    if (rc != DR_OK) return rc;
    rc = a.transposed ? ap_map(&mw, a.w, a.L, a.C, a.ldw, 64, 64) : ap_map(&mw, a.w, a.C, a.L, a.ldw, 64, wide ? 128 : cols);
    if (rc != DR_OK) return rc;
    //                                                    KPB PAIR  WIDE   ROWS  DUAL TERMS
    if (a.transposed) {
        if (wide) return ap_launch<ApKind<1, true, true, true, false, 2>>(mz, mw, p, overlap, smem, s);
        if (pair) return dual ? ap_launch<ApKind<1, true, false, true, true, 2>>(mz, mw, p, overlap, smem, s) : ap_launch<ApKind<1, true, false, true, false, 2>>(mz, mw, p, overlap, smem, s);
        if (kpb == 2) return dual ? ap_launch<ApKind<2, false, false, true, true, 2>>(mz, mw, p, overlap, smem, s) : ap_launch<ApKind<2, false, false, true, false, 2>>(mz, mw, p, overlap, smem, s);
        return dual ? ap_launch<ApKind<1, false, false, true, true, 2>>(mz, mw, p, overlap, smem, s) : ap_launch<ApKind<1, false, false, true, false, 2>>(mz, mw, p, overlap, smem, s);
    }
    if (wide) return f32 ? ap_launch<ApKind<1, true, true, false, false, 3>>(mz, mw, p, overlap, smem, s) : ap_launch<ApKind<1, true, true, false, false, 2>>(mz, mw, p, overlap, smem, s);
    if (pair) return f32 ? ap_launch<ApKind<1, true, false, false, false, 3>>(mz, mw, p, overlap, smem, s) : ap_launch<ApKind<1, true, false, false, false, 2>>(mz, mw, p, overlap, smem, s);
    if (kpb == 4) return f32 ? ap_launch<ApKind<4, false, false, false, false, 3>>(mz, mw, p, overlap, smem, s) : ap_launch<ApKind<4, false, false, false, false, 2>>(mz, mw, p, overlap, smem, s);
    if (kpb == 2) return f32 ? ap_launch<ApKind<2, false, false, false, false, 3>>(mz, mw, p, overlap, smem, s) : ap_launch<ApKind<2, false, false, false, false, 2>>(mz, mw, p, overlap, smem, s);
    return f32 ? ap_launch<ApKind<1, false, false, false, false, 3>>(mz, mw, p, overlap, smem, s) : ap_launch<ApKind<1, false, false, false, false, 2>>(mz, mw, p, overlap, smem, s);
}

}  // namespace dr
