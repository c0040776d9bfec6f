// The shared product with the adapters' second factors in the same accumulator, on the tensor cores (tcgen05, accumulators in TMEM):
//   out[m][c] = act(sum_l z[m][l] w[c][l] + bias[c] + sum_r T[m][r] f_a[c][r]),   T = scale_a factor t,  a the adapter of row m.
//
// A tile of 128 rows (256 by a pair of CTAs) may hold rows of many adapters.  Behind the blocks of 64 l it takes further
// blocks for the adapters in use among its rows, each with `rank` columns of its own: a row has its T in its adapter's columns and zeros in
// the others', so the same MMAs serve any mixture of requests, and the work grows with the adapters' bytes, which have to be read anyway.  T
// enters as the sum of two bfloat16 values (its columns twice, high and low), because a single one would cost the adapter's part 2^-9; of three
// where the result is float32.
// Where a mask lies between the adapter's product and the sum (the gradient of the input behind a dropout), that product has an accumulator of its own
// and the drain picks from it by the mask's bits.
//
// 0 * inf is NaN: entries of f that are not finite are 1 with their sign in these blocks, and what they add is added, for the rows of their own adapter
// only, in the drain.  Not 0: where T is infinite too the MMA would make NaN of an infinity; and where T is finite that drain makes the result an infinity
// or NaN, whatever the 1 has added.
//
// Bound by the tensor cores where l and the output are long (16384 x 4096 x 4096, rank 64: 370 us, 1.53 PFLOP/s, 0.94 of cuBLAS' rate), by the latencies of a tile's
// further blocks and drain where l is short (200704 x 64 x 256: 41 us, 3.5 a tile, of which memory 2).  The kernels of two accumulators spill 56 bytes a thread, transposed 88.
//
// 16 warps: 0 loads (TMA), 1 (and 2) issue MMAs, 4-11 drain, 12-15 find the rows' adapters and build the further blocks in the ring's
// stages.  A CTA's first tile takes them behind its blocks of l, so that w streams in while t is still being made; later tiles take them in front, so
// that they are built while the tile before is multiplied.
#include <algorithm>
#include <atomic>

#include "adapter.cuh"
#include "conv_common.cuh"
#include "umma_ptx.cuh"

namespace dr {
using namespace ptx;

constexpr int AP_THREADS = 512;
constexpr int AP_MAX_STAGES = 16;
constexpr int AP_SMEM = 180 * 1024;     // the ring's; with 32 KB of the drain's and the barriers' all of an SM's
constexpr int AP_SMEM_MOST = 213 * 1024;
constexpr int AP_TILE = 128;
// The tensor cores cut their sums off instead of rounding them: an error of about 1.5e-8 of the result for each MMA in a row, 4e-6 after 4096 l.  bfloat16
// results do not show it; for float32 ones 512 l (in the last or first sum the adapter's 3 rank columns too) are summed in TMEM at a time and the drain adds those up.
constexpr int AP_CHAIN = 8;             // blocks of 64 l

struct ApParams {
    AdRows rows;
    int L, C, R, Rp;
    uint32_t rp_magic;          // 2^32 / Rp, rounded up: columns / Rp by a multiplication
    int nt;                     // columns of a tile
    int tiles_c, tiles;
    int kblocks, stages;
    uint32_t a_bytes, b_bytes, stage_bytes;     // of a block of 64 l: z rows, w of this CTA; of a stage
    uint32_t acc_cols, tmem_cols;
    int split;                  // few rows: CTAs of a cluster that share a tile's l
    int accs;                   // few rows, float32 results: accumulators that share a CTA's l
    int early;                  // where in shared memory what they held before is added up
    int cache;                  // few rows: where T is kept in shared memory, 0: nowhere
    const int* row_id;
    const __nv_bfloat16* t;     // [M][terms][Rp]
    int t_terms;
    const float* bias;
    const __nv_bfloat16* f;
    size_t ldf;
    int f_vec;
    unsigned flags;
    void* out;
    size_t ldo;
    int out_vec;                // rows of the output on 16-byte boundaries
    const uint32_t* mask;       // DUAL: bits of what is kept, rows of ldm words
    int ldm;
    int* status;
};

struct ApShared {
    uint64_t full[AP_MAX_STAGES], empty[AP_MAX_STAGES], tfull[2], tempty[2], ifull[3], iempty[3], loads[3], built[3];
    uint32_t tmem;
    int abort;
    // what the builders find out about a tile: kept for three of them, one being drained, one multiplied, one looked at ahead
    int ext[3];                 // columns of T of the tile
    int odd[3];                 // number (from 1) of the latest tile that met an f that is not finite
    int slot[3][AP_TILE];       // place of the row's adapter in list, ROW_SHARED or ROW_NONE
    uint16_t list[3][2 * AP_TILE];
    alignas(16) float bias[3][512];
    ApFind find;
};
// a place in that ring of three and how often it was used
struct ApInfo {
    int at = 0;
    uint32_t use = 0;
    __device__ __forceinline__ void next() { if (++at == 3) { at = 0; use ^= 1; } }
};

__device__ __forceinline__ uint32_t sdesc_rows_lo(uint32_t smem_addr, uint32_t box) {    // contraction index = row of a 64-column box
    return ((smem_addr & 0x3FFFFu) >> 4) | (((box >> 4) & 0x3FFFu) << 16);
}
__device__ __forceinline__ void st_shared16(uint32_t addr, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// bits 15 and 31 of the result are set where a half of u has an exponent of all ones
__device__ __forceinline__ uint32_t odd_halves(uint32_t u) { return (u & 0x7FFF7FFFu) + 0x00800080u; }
template <int N>
__device__ __forceinline__ bool any_odd(const uint4 (&v)[N]) {
    uint32_t o = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) o |= odd_halves(v[i].x) | odd_halves(v[i].y) | odd_halves(v[i].z) | odd_halves(v[i].w);
    return (o & 0x80008000u) != 0;
}
// entries that are not finite become 1 with their sign
__device__ __forceinline__ uint32_t finite_halves(uint32_t u) {
    const uint32_t odd = ((odd_halves(u) & 0x80008000u) >> 15) * 0x7FFFu;
    return (u & ~odd) | (odd & 0x3F803F80u);
}

// What one kernel is compiled for.  PAIR: tiles of 256 rows by two CTAs.  WIDE (pairs): two accumulators of 256
// columns share the rows' blocks, each with an issuing warp of its own.  ROWS: w and f have the contraction index as their rows.  DUAL: an
// accumulator of its own for the adapters.  TERMS: bfloat16 values to a T.
template <bool PAIR_, bool WIDE_, bool ROWS_, bool DUAL_, int TERMS_>
struct ApKind {
    static constexpr int TERMS = TERMS_;
    static constexpr bool PAIR = PAIR_, WIDE = WIDE_, ROWS = ROWS_, DUAL = DUAL_;
    static constexpr int WIDTH = TERMS == 2 ? 32 : 16;         // columns of T in a further block of 64
    static constexpr int EACH = PAIR && !WIDE ? 4 : 8;          // 16-byte pieces of a block's f that a thread brings, at most
};

// ---- the builders' steps (128 threads, bt their number) --------------------------------------------------------------------
// eight values of a row whose rank leaves them no alignment, zeros behind the last
__device__ __noinline__ uint4 ap_odd_rank(const __nv_bfloat16* src, int n) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = 2 * i < n ? __ldg(reinterpret_cast<const unsigned short*>(src) + 2 * i) : 0u;
        u[i] = lo | (2 * i + 1 < n ? (uint32_t)__ldg(reinterpret_cast<const unsigned short*>(src) + 2 * i + 1) << 16 : 0u);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// This thread's pieces of f in the block of `eb`: rows row0 + i * step of the block (ROWS: contraction rows, else columns of the output), 16 bytes at cj;
// column(i): the output column that place i of the CTA's is.
template <class Kind, class Column>
__device__ __forceinline__ void ap_load_f(const ApParams& p, const uint16_t* list, int eb, int w, int cols, int row0, int step, int cj, Column column, uint4 (&fv)[Kind::EACH]) {
    const int ef = eb + 8 * cj, df = (int)__umulhi((uint32_t)ef, p.rp_magic), rf = ef - df * p.Rp;
    const bool mine = Kind::ROWS || 8 * cj < w;
    const int c_rows = Kind::ROWS ? column(8 * cj) : 0;
    const __nv_bfloat16* fa = p.f + (Kind::ROWS ? (size_t)c_rows : mine ? (size_t)list[df] * p.C * p.R + rf : 0);
#pragma unroll
    for (int i = 0; i < Kind::EACH; ++i) {
        fv[i] = make_uint4(0, 0, 0, 0);
        const int row = row0 + i * step;
        if (Kind::ROWS) {
            if (row < w && c_rows < p.C) {
                const int e = eb + row, d = (int)__umulhi((uint32_t)e, p.rp_magic), r = e - d * p.Rp;
                if (r < p.R) fv[i] = __ldg(reinterpret_cast<const uint4*>(fa + ((size_t)list[d] * p.R + r) * p.ldf));
            }
        } else {
            const int c = column(row);
            if (mine && row < cols && c < p.C) {
                const __nv_bfloat16* src = fa + (size_t)c * p.R;
                fv[i] = p.f_vec ? __ldg(reinterpret_cast<const uint4*>(src)) : ap_odd_rank(src, p.R - rf);
            }
        }
    }
}
// T of this thread's row (in global or shared memory) in the block of `eb`, eight columns at a time
template <class Kind>
__device__ __forceinline__ void ap_load_t(const __nv_bfloat16* trow, int slot, int Rp, int eb, int w, uint4 (&tv)[Kind::WIDTH / 8][Kind::TERMS]) {
#pragma unroll
    for (int j = 0; j < Kind::WIDTH / 8; ++j) {
        const int r = eb + 8 * j - slot * Rp;
        const bool there = slot >= 0 && (unsigned)r < (unsigned)Rp && 8 * j < w;
#pragma unroll
        for (int k = 0; k < Kind::TERMS; ++k) tv[j][k] = there ? *reinterpret_cast<const uint4*>(trow + k * Rp + r) : make_uint4(0, 0, 0, 0);
    }
}
// both into the stage: z's part at a (rows of 128 bytes), w's at b
template <class Kind>
__device__ __forceinline__ void ap_store_block(uint32_t a, uint32_t b, int bt, bool row_there, int w, int cols, int row0, int step, int cj, const uint4 (&fv)[Kind::EACH],
                                               const uint4 (&tv)[Kind::WIDTH / 8][Kind::TERMS]) {
    const int wc = w >> 3;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    if (row_there) {
        const uint32_t at = a + bt * 128, x = (uint32_t)(bt & 7);
#pragma unroll
        for (int i = 0; i < Kind::WIDTH / 8; ++i)
            if (i < wc) {
#pragma unroll
                for (int k = 0; k < Kind::TERMS; ++k) st_shared16(at + (((uint32_t)(i + k * wc) ^ x) << 4), tv[i][k]);
            }
        if (Kind::TERMS == 3 && wc == 1) st_shared16(at + ((3u ^ x) << 4), zero);              // 24 columns: two steps of 16
    }
#pragma unroll
    for (int i = 0; i < Kind::EACH; ++i) {
        const int row = row0 + i * step;
        if (Kind::ROWS) {
            if (row < w) {
                const uint32_t g = b + (uint32_t)(cj >> 3) * 8192u;
#pragma unroll
                for (int k = 0; k < Kind::TERMS; ++k) st_shared16(g + (row + k * w) * 128 + (((cj & 7) ^ ((row + k * w) & 7)) << 4), fv[i]);
            }
        } else if (row < cols && cj < wc) {
            const uint32_t at = b + row * 128, x = (uint32_t)(row & 7);
#pragma unroll
            for (int k = 0; k < Kind::TERMS; ++k) st_shared16(at + (((uint32_t)(cj + k * wc) ^ x) << 4), fv[i]);
            if (Kind::TERMS == 3 && wc == 1) st_shared16(at + ((3u ^ x) << 4), zero);
        }
    }
}
// what entries of f that are not finite add to out[m][c]: an infinity, NaN, or 0
template <bool ROWS>
__device__ __noinline__ float ap_odd(const ApParams& p, int a, int m, int c) {
    float s = 0.f;
    for (int r = 0; r < p.R; ++r) {
        const float fr = __bfloat162float(ROWS ? p.f[((size_t)a * p.R + r) * p.ldf + c] : p.f[((size_t)a * p.C + c) * p.R + r]);
        if (fabsf(fr) <= 3.4e38f) continue;
        const __nv_bfloat16* t = p.t + (size_t)m * p.t_terms * p.Rp + r;
        s = fmaf(__bfloat162float(__ldcg(t)) + __bfloat162float(__ldcg(t + p.Rp)), fr, s);
    }
    return s;
}
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
adapter_product_kernel(const __grid_constant__ CUtensorMap map_z, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_out,
                       const __grid_constant__ ApParams p) {
    constexpr bool PAIR = Kind::PAIR, WIDE = Kind::WIDE, ROWS = Kind::ROWS, DUAL = Kind::DUAL;
    constexpr int TERMS = Kind::TERMS, WIDTH = Kind::WIDTH;
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
    const uint32_t stage_out = ring + (uint32_t)p.stages * p.stage_bytes;      // after the ring, 4 KB for each draining warp
    auto further_stages = [](int ext) { return (ext + Kind::WIDTH - 1) / Kind::WIDTH; };

    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { mbar_init(&sh.full[i], PAIR ? 2 : 1); mbar_init(&sh.empty[i], WIDE ? 2 : 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.tfull[i], 1);
            mbar_init(&sh.tempty[i], PAIR ? 16 : 8);
        }
        for (int i = 0; i < 3; ++i) {
            mbar_init(&sh.loads[i], 1);
            mbar_init(&sh.built[i], 1);
            mbar_init(&sh.ifull[i], 128);
            mbar_init(&sh.iempty[i], 9 + (rank == 0 ? (WIDE ? 2 : 1) : 0));
            sh.odd[i] = 0;
        }
        sh.abort = 0;
        fence_barrier_init();
        prefetch_tensormap(&map_z);
        prefetch_tensormap(&map_w);
        if (p.out_vec) prefetch_tensormap(&map_out);
    }
    if (warp == 1) {
        if (PAIR) { tmem_alloc_pair(&sh.tmem, p.tmem_cols); tmem_relinquish_pair(); }
        else { tmem_alloc(&sh.tmem, p.tmem_cols); tmem_relinquish(); }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    grid_launch_dependents();
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
            ApInfo info;
            // Passes over the further blocks of a tile.  The parity of a barrier tells two neighbouring phases apart and no more: who waits for a stage
            // must know that the use before the last one is over, and no barrier here may run two phases ahead of one who waits for it (three of each are
            // enough: no one is further ahead than the builders, who look at a tile while the one three in front of it is done).  The builders know it once the loads in front of theirs are all
            // issued (sh.loads); this thread where the further blocks since its last load are fewer than the stages, and otherwise once they are
            // built.
            auto pass = [&](int tile) {
                if (!mbar_wait(&sh.ifull[info.at], info.use, abort_flag)) { give_up(82, tile); return false; }
                const int further = further_stages(sh.ext[info.at]);
                mbar_arrive(&sh.iempty[info.at]);
                gap += further;
                if (it > 0 && gap >= p.stages && !mbar_wait(&sh.built[info.at], info.use, abort_flag)) { give_up(91, tile); return false; }
                info.next();
                s += further;
                while (s >= p.stages) { s -= p.stages; ph ^= 1; }
                return true;
            };
            for (int tile = unit; tile < p.tiles && ok; tile += units, ++it) {
                const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c;
                const int m0 = mt * tile_m + (int)rank * AP_TILE, c0 = ct * p.nt;
                if (it > 0 && !pass(tile)) break;
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    if (!mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag)) { give_up(81, tile); ok = false; break; }
                    const uint32_t fb = (full0 + 8 * s) & full_mask;
                    if (!PAIR || rank == 0) mbar_expect_tx_u32(fb, (PAIR ? 2u : 1u) * p.stage_bytes);
                    const uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + p.a_bytes;
                    const int l = kb << 6;
                    tma_load_2d_u32<PAIR>(a, &map_z, fb, l, m0, 1u);
                    if (ROWS) {
                        for (int g = 0; g < cols >> 6; ++g) tma_load_2d_u32<PAIR>(b + (uint32_t)g * 8192u, &map_w, fb, c0 + column(64 * g), l, 1u);
                    } else {
                        tma_load_2d_u32<PAIR>(b, &map_w, fb, l, c0 + column(0), 1u);
                        if (WIDE) tma_load_2d_u32<PAIR>(b + 16384u, &map_w, fb, l, c0 + column(128), 1u);
                    }
                    if (PAIR && rank == 0) mbar_arrive(&sh.full[s]);      // the barrier counts two: in a further block each CTA's builders
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!ok) break;
                gap = 0;
                mbar_arrive(&sh.loads[it % 3]);
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
            ApInfo info;
            auto further = [&](int tile) {
                if (!mbar_wait(&sh.ifull[info.at], info.use, abort_flag)) { give_up(85, tile); return false; }
                const int ext = sh.ext[info.at];
                mbar_arrive(&sh.iempty[info.at]);
                info.next();
                const uint32_t de = d + (DUAL ? p.acc_cols : 0u);
                uint32_t acc = DUAL ? 0u : accum;
                for (int e = 0; e < ext; e += WIDTH) {
                    if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(86, tile); return false; }
                    tc_fence_after();
                    const uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + p.a_bytes + (uint32_t)half * 16384u;
                    const int n16 = (TERMS * min(WIDTH, ext - e) + 15) >> 4;
                    const uint32_t al = sdesc_lo(a), bl = ROWS ? sdesc_rows_lo(b, 8192) : sdesc_lo(b);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        umma_bf16_lo<PAIR>(de, al + 2 * k, bl + b_step * k, idesc, acc, k < n16 ? 1u : 0u);
                        acc = 1;
                    }
                    umma_commit_u32<PAIR>(empty0 + 8 * s);
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!DUAL) accum = acc;
                return true;
            };
            int n = 0;                                                          // accumulators begun
            for (int tile = unit; tile < p.tiles; tile += units, ++it) {
                auto begin = [&]() {                                            // the next accumulator, once it is drained
                    const int ab = WIDE ? half : n & 1, use = WIDE ? n : n >> 1;
                    if (!mbar_wait(&sh.tempty[ab], (use & 1) ^ 1, abort_flag)) { give_up(83, tile); return false; }
                    tc_fence_after();
                    d = tmem + (uint32_t)ab * p.acc_cols * (DUAL ? 2u : 1u);
                    accum = 0;
                    return true;
                };
                auto end = [&]() { umma_commit_u32<PAIR>(smem_u32(&sh.tfull[WIDE ? half : n & 1])); ++n; };
                if (!begin()) break;
                if (it > 0 && !further(tile)) break;
                bool ok = true;
                for (int kb = 0; kb < p.kblocks; ++kb) {
                    if (TERMS == 3 && kb > 0 && kb % AP_CHAIN == 0) {
                        end();
                        if (!begin()) { ok = false; break; }
                    }
                    if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(84, tile); ok = false; break; }
                    tc_fence_after();
                    const uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + p.a_bytes + (uint32_t)half * 16384u;
                    const uint32_t al = sdesc_lo(a), bl = ROWS ? sdesc_rows_lo(b, 8192) : sdesc_lo(b);
                    const int n16 = kb == p.kblocks - 1 ? tail16 : 4;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        umma_bf16_lo<PAIR>(d, al + 2 * k, bl + b_step * k, idesc, accum, k < n16 ? 1u : 0u);
                        accum = 1;
                    }
                    umma_commit_u32<PAIR>(empty0 + 8 * s);
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                if (!ok || (it == 0 && !further(tile))) break;
                end();
            }
        }
        __syncwarp();
    } else if (warp >= 12) {
        // ---------------------------------------------------------------- the rows' adapters, and the further blocks
        const int bt = threadIdx.x - 384;
        constexpr int H = PAIR ? 2 : 1;
        const int cpr = ROWS ? cols >> 3 : 4;                                  // 16-byte pieces of a row of a block
        const int cj = bt % cpr, row0 = bt / cpr, step = 128 / cpr;
        struct Opened { int it, at, ext, slot, c0; const __nv_bfloat16* trow; };   // a tile that has been looked at
        struct Block { uint4 f[Kind::EACH]; };
        int id[H];
        auto ids = [&](int tile) {
            const int mt = tile / p.tiles_c;
#pragma unroll
            for (int h = 0; h < H; ++h) {
                const int m = mt * tile_m + h * AP_TILE + bt;
                id[h] = tile < p.tiles && m < p.rows.M ? __ldcg(p.row_id + m) : ROW_NONE;
            }
        };
        ApInfo info;
        // looks at a tile, whose rows' adapters are in id[], and tells the others; false: a wait ran out
        auto open = [&](int tile, int it, Opened& o) {
            const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c;
            o.it = it;
            o.at = info.at;
            o.c0 = ct * p.nt;
            const bool free_now = mbar_wait(&sh.iempty[info.at], info.use ^ 1, abort_flag);
            if (!free_now) give_up(87, tile);
            if (builders_any(!free_now)) return false;
            if (p.flags & DR_BIAS)
                for (int c = bt; c < p.nt; c += 128) sh.bias[info.at][c] = o.c0 + c < p.C ? __ldg(p.bias + o.c0 + c) : 0.f;
            int slots[H];
            o.ext = ap_find(sh.find, sh.list[info.at], id, slots, bt) * p.Rp;
            o.slot = slots[PAIR ? rank : 0];
            o.trow = p.t + (size_t)(mt * tile_m + (int)rank * AP_TILE + bt) * p.t_terms * p.Rp;
            sh.slot[info.at][bt] = o.slot;
            if (bt == 0) sh.ext[info.at] = o.ext;
            ids(tile + units);                          // the next tile's on their way
            builders_sync();                            // the list stands; and no one still reads what the next search clears
            mbar_arrive(&sh.ifull[info.at]);
            info.next();
            return true;
        };
        auto load = [&](const Opened& o, int e0, Block& k) {
            const int w = min(WIDTH, o.ext - e0);
            ap_load_f<Kind>(p, sh.list[o.at], e0, w, cols, row0, step, cj, [&](int i) { return o.c0 + column(i); }, k.f);
        };
        int s = 0;
        uint32_t ph = 0;
        auto advance = [&](int n) {
            s += n;
            while (s >= p.stages) { s -= p.stages; ph ^= 1; }
        };
        auto store = [&](const Opened& o, int e0, Block& k, const uint4 (&tv)[WIDTH / 8][TERMS]) {
            if (any_odd(k.f)) {
#pragma unroll
                for (int i = 0; i < Kind::EACH; ++i) k.f[i] = make_uint4(finite_halves(k.f[i].x), finite_halves(k.f[i].y), finite_halves(k.f[i].z), finite_halves(k.f[i].w));
                // Both CTAs of a pair drain all columns: each is told.  The number only grows, so that a CTA that runs ahead hides nothing
                // from one behind; a number ahead of a tile's costs that tile a search for entries it does not have.
                if (PAIR) {
                    for (uint32_t c = 0; c < 2; ++c)
                        asm volatile("red.relaxed.cluster.shared::cluster.max.s32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&sh.odd[o.at]), c)), "r"(o.it + 1) : "memory");
                } else {
                    atomicMax(&sh.odd[o.at], o.it + 1);
                }
            }
            const int before = o.it == 0 ? 0 : o.it - 1;                       // the tile whose loads lie in front of this block
            const bool slot_free = __all_sync(0xffffffffu, mbar_wait(&sh.loads[before % 3], (uint32_t)(before / 3) & 1, abort_flag) && mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag));
            if (!slot_free) give_up(88, o.it);
            if (slot_free) {
                const uint32_t a = ring + (uint32_t)s * p.stage_bytes;
                ap_store_block<Kind>(a, a + p.a_bytes, bt, true, min(WIDTH, o.ext - e0), cols, row0, step, cj, k.f, tv);
            }
            fence_proxy_async_smem();
            if (builders_any(!slot_free)) return false;
            if (bt == 0) {
                if (PAIR) mbar_arrive_leader(&sh.full[s]);
                else mbar_arrive(&sh.full[s]);
            }
            advance(1);
            return true;
        };
        grid_dependency_wait();                                                // the rows' adapters, and t, are the kernel's in front
        ids(unit);
        Opened now;
        bool ok = unit < p.tiles && open(unit, 0, now);
        for (int tile = unit, it = 0; ok && tile < p.tiles; tile += units, ++it) {
            if (it == 0) advance(p.kblocks);
            // A block's loads go out once the one in front of it is handed over: a fence waits for what is on its way, and the next block's loads in front of
            // it cost more than they hid: 200704 x 64 x 256 69 us, so 65
#pragma unroll 1
            for (int e0 = 0; ok && e0 < now.ext; e0 += WIDTH) {
                Block block;
                uint4 tv[WIDTH / 8][TERMS];
                ap_load_t<Kind>(now.trow, now.slot, p.Rp, e0, min(WIDTH, now.ext - e0), tv);
                load(now, e0, block);
                ok = store(now, e0, block, tv);
            }
            if (!ok) break;
            if (bt == 0) mbar_arrive(&sh.built[now.at]);
            if (it > 0) advance(p.kblocks);
            if (tile + units < p.tiles) ok = open(tile + units, it + 1, now);
        }
    } else if (warp >= 4) {
        // ---------------------------------------------------------------- drain: two warps to a quarter of the rows, every other 128 bytes of columns each
        const int q = warp & 3, side = (warp - 4) >> 2;
        const uint32_t buf = stage_out + (uint32_t)(warp - 4) * 4096u;
        const uint32_t put = buf + lane * 128, px = (uint32_t)(lane & 7);
        const bool f32 = TERMS == 3;
        constexpr int CHUNK = TERMS == 3 ? 32 : 64;                            // columns of 128 bytes
        const float low = (p.flags & DR_RELU) ? 0.f : -INFINITY;
        const uint32_t low2 = (p.flags & DR_RELU) ? 0u : 0xFF80FF80u;
        int it = 0, n = 0;
        bool ok = true;
        ApInfo info;
        for (int tile = unit; tile < p.tiles && ok; tile += units, ++it, info.next()) {
            const int ib = info.at;
            const int mt = tile / p.tiles_c, ct = tile - mt * p.tiles_c;
            const int n0 = ct * p.nt, n_here = min(p.nt, p.C - n0);
            if (!__all_sync(0xffffffffu, mbar_wait(&sh.ifull[ib], info.use, abort_flag))) { give_up(89, tile); break; }
            const int slot = sh.slot[ib][q * 32 + lane];
            const unsigned valid = __ballot_sync(0xffffffffu, slot != ROW_NONE);
            const int mw = mt * tile_m + (int)rank * AP_TILE + q * 32, m = mw + lane;
            const int ext = sh.ext[ib];
            // no row of no request among them: whole boxes by TMA, which leaves out what lies behind the last row or column
            const bool boxes = p.out_vec && mw < p.rows.M && valid == (p.rows.M - mw >= 32 ? 0xffffffffu : (1u << (p.rows.M - mw)) - 1u);
            const uint32_t quarter = (uint32_t)(q * 32) << 16;
#pragma unroll 1
            for (int part = 0; part < (WIDE ? 2 : 1); ++part) {
                // float32 results: this warp's columns, at most two chunks (nt <= 128), added up over the chains in front of the last
                float sum[TERMS == 3 ? 2 : 1][32];
                if (TERMS == 3) {
#pragma unroll
                    for (int j = 0; j < 2; ++j)
#pragma unroll
                        for (int i = 0; i < 32; ++i) sum[TERMS == 3 ? j : 0][i] = 0.f;
                    for (int kb = AP_CHAIN; kb < p.kblocks; kb += AP_CHAIN, ++n) {
                        if (!__all_sync(0xffffffffu, mbar_wait(&sh.tfull[n & 1], (uint32_t)(n >> 1) & 1, abort_flag))) { give_up(90, tile); ok = false; break; }
                        tc_fence_after();
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            if (side * 32 + 64 * j >= n_here) break;
                            uint32_t v[32];
                            tmem_ld_x32(tmem + (uint32_t)(n & 1) * p.acc_cols + quarter + side * 32 + 64 * j, v);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; ++i) sum[TERMS == 3 ? j : 0][i] += __uint_as_float(v[i]);
                        }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) {
                            if (PAIR) mbar_arrive_leader(&sh.tempty[n & 1]);
                            else mbar_arrive(&sh.tempty[n & 1]);
                        }
                    }
                    if (!ok) break;
                }
                uint2 kept = make_uint2(0, 0);                                 // of this warp's 64 columns: DUAL tiles have at most 128
                if (DUAL && ext && m < p.rows.M && n0 + 64 * side < p.C) kept = __ldcg(reinterpret_cast<const uint2*>(p.mask + (size_t)m * p.ldm + (n0 >> 5)) + side);
                const int ab = WIDE ? part : n & 1, use = WIDE ? it : n >> 1;
                if (!__all_sync(0xffffffffu, mbar_wait(&sh.tfull[ab], use & 1, abort_flag))) { give_up(90, tile); ok = false; break; }
                tc_fence_after();
                const bool odd = *(volatile int*)&sh.odd[ib] > it;
                const uint32_t acc = tmem + (uint32_t)ab * p.acc_cols * (DUAL ? 2u : 1u) + quarter;
                const int c_end = WIDE ? min(256, n_here - 256 * part) : n_here, cb = WIDE ? 256 * part : 0;
#pragma unroll(TERMS == 3 ? 2 : 1)
                for (int cj = 0; cj < (TERMS == 3 ? 2 : 1 << 30); ++cj) {
                    const int c = (side + 2 * cj) * CHUNK;
                    if (c >= c_end) break;
                    if (lane == 0) tma_store_wait_read();                      // the box in front has been read
                    __syncwarp();
                    uint32_t w[DUAL ? 1 : CHUNK / 32][32];
                    if (!DUAL) {
#pragma unroll
                        for (int h = 0; h < CHUNK / 32; ++h) tmem_ld_x32(acc + c + 32 * h, w[h % (DUAL ? 1 : CHUNK / 32)]);
                    }
#pragma unroll(DUAL ? 1 : CHUNK / 32)
                    for (int h = 0; h < CHUNK; h += 32) {                      // rolled where it is long: the code has to stay in the instruction cache
                        uint32_t (&v)[32] = w[DUAL ? 0 : h / 32];
                        if (DUAL) tmem_ld_x32(acc + c + h, v);
                        const uint32_t bits = h ? kept.y : kept.x;
                        if (DUAL && ext) {
                            uint32_t u[32];
                            tmem_ld_x32(acc + p.acc_cols + c + h, u);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + (bits >> i & 1 ? __uint_as_float(u[i]) : 0.f));
                        }
                        tmem_ld_wait();
                        if (TERMS == 3) {
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + sum[TERMS == 3 ? cj & 1 : 0][i]);
                        }
                        if (odd) {
                            // what f that is not finite adds to this row's values
#pragma unroll 1
                            for (int i = 0; i < 32; ++i) {
                                const int col = n0 + cb + c + h + i;
                                const bool mine = slot >= 0 && col < p.C && (!DUAL || (bits >> i & 1));
                                const float x = mine ? ap_odd<ROWS>(p, sh.list[ib][slot], m, col) : 0.f;
#pragma unroll
                                for (int k = 0; k < 32; ++k)
                                    if (k == i && x != 0.f) v[k] = __float_as_uint(__uint_as_float(v[k]) + x);
                            }
                        }
                        if (p.flags & DR_BIAS) {
                            const float4* bias = reinterpret_cast<const float4*>(&sh.bias[ib][cb + c + h]);
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float4 x = bias[i];
                                v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + x.x);
                                v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + x.y);
                                v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + x.z);
                                v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + x.w);
                            }
                        }
                        // through shared memory, so that whole rows of 128 bytes are written
                        if (f32) {
#pragma unroll
                            for (int j = 0; j < 8; ++j)
                                st_shared16(put + (((uint32_t)j ^ px) << 4),
                                            make_uint4(__float_as_uint(max_nan(__uint_as_float(v[4 * j]), low)), __float_as_uint(max_nan(__uint_as_float(v[4 * j + 1]), low)),
                                                       __float_as_uint(max_nan(__uint_as_float(v[4 * j + 2]), low)), __float_as_uint(max_nan(__uint_as_float(v[4 * j + 3]), low))));
                        } else {
#pragma unroll
                            for (int j = 0; j < 4; ++j) {
                                const float* y = reinterpret_cast<const float*>(v + 8 * j);
                                st_shared16(put + (((uint32_t)(j + (h >> 3)) ^ px) << 4),
                                            make_uint4(max_nan_bf16x2(pack_bf16(y[0], y[1]), low2), max_nan_bf16x2(pack_bf16(y[2], y[3]), low2),
                                                       max_nan_bf16x2(pack_bf16(y[4], y[5]), low2), max_nan_bf16x2(pack_bf16(y[6], y[7]), low2)));
                            }
                        }
                    }
                    if (boxes && (c_end - c >= CHUNK || (n0 + cb + c_end == p.C && p.C * (f32 ? 4 : 2) % 16 == 0))) {
                        fence_proxy_async_smem();
                        __syncwarp();
                        if (lane == 0) {
                            tma_store_2d(&map_out, buf, (n0 + cb + c) * (f32 ? 2 : 1), mw);      // float32 go as pairs of 16 bits
                            tma_store_commit();
                        }
                        continue;
                    }
                    __syncwarp();
                    const int have = min(CHUNK, c_end - c);
#pragma unroll 1
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
                    __syncwarp();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) mbar_arrive_leader(&sh.tempty[ab]);
                    else mbar_arrive(&sh.tempty[ab]);
                }
            }
            ++n;
            if (lane == 0) mbar_arrive(&sh.iempty[ib]);
        }
        if (lane == 0) tma_store_wait_all();
    }
    tc_fence_before();
    ap_settle(abort_flag);
    if (PAIR) cluster_sync_all();
    if (warp == 1) {
        if (PAIR) tmem_dealloc_pair(tmem, p.tmem_cols);
        else tmem_dealloc(tmem, p.tmem_cols);
    }
}

// ---- few rows (one tile of at most 128) ------------------------------------------------------------------------------------------------
// Bound by the bytes of w, and by latency.  A cluster of CTAs shares a tile's l: each takes a range of it and every so many of the further blocks, and the
// accumulators meet in distributed shared memory, where each CTA sums and finishes a part of the columns.  Rows of z behind the last are not
// loaded: what the MMA finds there only reaches rows of the accumulator that nobody reads.  8 warps of at most 128 registers (0 loads, 1 issues MMAs, 4-7
// build the further blocks and then drain), so that a CTA fits beside the first product's and w streams in while t is still being made.
//
// float32 results: sums of at most 512 l, each in the next accumulator.  Where a CTA has more of them than accumulators, the builders first add the ones in front
// up in shared memory: the further blocks are multiplied last, so nobody waits for one who waits for them.  128 x 32768 x 9472 (rank 16) in sums
// of 8192 was off by 2.3e-6, and is by 5.7e-7; 206 us, and 208 so.
constexpr int AP_FEW_THREADS = 256;
// Two CTAs fit an SM whatever they hold of its tensor memory: 256 columns each, registers for no third, and shared memory for none either however few
// registers a compiler takes.  A third would wait for tensor memory while its cluster's others hold theirs, and clusters might wait for one another.
constexpr int AP_FEW_ACCS = 8;
constexpr int AP_FEW_SMEM = 80 * 1024;
struct ApFewShared {
    uint64_t full[AP_MAX_STAGES], empty[AP_MAX_STAGES], cfull[AP_FEW_ACCS], cempty[AP_FEW_ACCS], tfull, loads, ifull;
    uint32_t tmem;
    int abort, odd, ext;
    int slot[AP_TILE];
    uint16_t list[AP_TILE];
    ApFind find;
    float bias[AP_TILE];        // of the columns this CTA finishes
};

template <class Kind>
__global__ void __launch_bounds__(AP_FEW_THREADS, 2)
adapter_few_kernel(const __grid_constant__ CUtensorMap map_z, const __grid_constant__ CUtensorMap map_w, const __grid_constant__ ApParams p) {
    constexpr bool ROWS = Kind::ROWS, DUAL = Kind::DUAL;
    constexpr int TERMS = Kind::TERMS, WIDTH = Kind::WIDTH;
    extern __shared__ uint8_t ap_raw[];
    __shared__ ApFewShared sh;
    const uint32_t ring = (smem_u32(ap_raw) + 1023u) & ~1023u;
    float* const sums = reinterpret_cast<float*>(ap_raw + (ring - smem_u32(ap_raw)));      // once the ring is done: [M][nt + 4], DUAL: the adapters' behind
    __nv_bfloat16* const cache = reinterpret_cast<__nv_bfloat16*>(ap_raw + (ring - smem_u32(ap_raw)) + p.cache);       // behind the ring
    const int pitch = p.nt + 4;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = p.split > 1 ? (int)cluster_ctarank() : 0;
    const int tile = (int)blockIdx.x / p.split, c0 = tile * p.nt;
    const int kb0 = (int)((long long)rank * p.kblocks / p.split), kb1 = (int)((long long)(rank + 1) * p.kblocks / p.split);
    volatile int* abort_flag = &sh.abort;
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < AP_FEW_ACCS; ++i) { mbar_init(&sh.cfull[i], 1); mbar_init(&sh.cempty[i], 4); }
        mbar_init(&sh.tfull, 1);
        mbar_init(&sh.loads, 1);
        mbar_init(&sh.ifull, 128);
        sh.abort = 0;
        sh.odd = 0;
        fence_barrier_init();
        prefetch_tensormap(&map_z);
        prefetch_tensormap(&map_w);
    }
    if (warp == 1) { tmem_alloc(&sh.tmem, p.tmem_cols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    if (p.split > 1) cluster_sync_all();                       // sh.odd of every CTA stands before another one writes it
    tc_fence_after();
    grid_launch_dependents();
    const uint32_t tmem = sh.tmem;
    const uint32_t full0 = smem_u32(&sh.full[0]), empty0 = smem_u32(&sh.empty[0]);
    auto give_up = [&](int site) {
        if (!*abort_flag) report_timeout(p.status, site, tile);
        *abort_flag = 1;
    };

    // float32 results: sums of `chain` blocks, each in the next accumulator; of more of them than there are accumulators, the ones in front are drained early
    const int chain = TERMS == 3 ? min(AP_CHAIN, (kb1 - kb0 + p.accs - 1) / p.accs) : 1 << 30;
    const int chains = TERMS == 3 ? (kb1 - kb0 + chain - 1) / chain : 1, early = chains - p.accs;

    if (warp == 0) {
        if (lane == 0) {
            int s = 0;
            uint32_t ph = 0;
            for (int kb = kb0; kb < kb1; ++kb) {
                if (!mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag)) { give_up(92); break; }
                const uint32_t fb = full0 + 8 * s;
                mbar_expect_tx_u32(fb, p.stage_bytes);
                const uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + p.a_bytes;
                const int l = kb << 6;
                if (ROWS) {
                    for (int g = 0; g < p.nt >> 6; ++g) tma_load_2d_u32<false>(b + (uint32_t)g * 8192u, &map_w, fb, c0 + 64 * g, l, 1u);
                } else {
                    tma_load_2d_u32<false>(b, &map_w, fb, l, c0, 1u);
                }
                tma_load_2d_u32<false>(a, &map_z, fb, l, 0, 1u);
                if (++s == p.stages) { s = 0; ph ^= 1; }
            }
            mbar_arrive(&sh.loads);
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = make_idesc_bf16(AP_TILE, p.nt) | (ROWS ? 1u << 16 : 0u);
            const int tail16 = ((p.L - ((p.kblocks - 1) << 6)) + 15) >> 4;
            constexpr uint32_t b_step = ROWS ? 128u : 2u;
            int s = 0;
            uint32_t ph = 0, accum = 0;
            bool ok = true;
            auto block = [&](uint32_t d, int n16, int site) {
                if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(site); ok = false; return; }
                tc_fence_after();
                const uint32_t a = ring + (uint32_t)s * p.stage_bytes, b = a + p.a_bytes;
                const uint32_t al = sdesc_lo(a), bl = ROWS ? sdesc_rows_lo(b, 8192) : sdesc_lo(b);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    umma_bf16_lo<false>(d, al + 2 * k, bl + b_step * k, idesc, accum, k < n16 ? 1u : 0u);
                    accum = 1;
                }
                umma_commit_u32<false>(empty0 + 8 * s);
                if (++s == p.stages) { s = 0; ph ^= 1; }
            };
            int acc = 0, use = 0;                                               // the chain's accumulator, and how often that was used
            for (int kb = kb0, c = 0; ok; ++c) {
                const int end = TERMS == 3 ? min(kb1, kb + chain) : kb1;
                if (TERMS == 3 && use > 0) {
                    if (!mbar_wait(&sh.cempty[acc], (uint32_t)(use - 1) & 1, abort_flag)) { give_up(99); ok = false; break; }
                    tc_fence_after();
                }
                accum = 0;
                const uint32_t d = tmem + (TERMS == 3 ? (uint32_t)acc * p.acc_cols : 0u);
#pragma unroll 1
                for (; kb < end && ok; ++kb) block(d, kb == p.kblocks - 1 ? tail16 : 4, 93);
                if (kb >= kb1) break;
                if (TERMS == 3) {
                    if (c < early) umma_commit_u32<false>(smem_u32(&sh.cfull[acc]));
                    if (++acc == p.accs) { acc = 0; ++use; }
                }
            }
            if (ok && !mbar_wait(&sh.ifull, 0, abort_flag)) { give_up(94); ok = false; }
            const int ext = ok ? sh.ext : 0;
            if (DUAL) accum = 0;
            const uint32_t last = TERMS == 3 ? (uint32_t)acc * p.acc_cols : 0u;
            for (int e = rank * WIDTH; e < ext && ok; e += p.split * WIDTH) block(tmem + (DUAL ? p.acc_cols : last), (TERMS * min(WIDTH, ext - e) + 15) >> 4, 95);
            umma_commit_u32<false>(smem_u32(&sh.tfull));
        }
        __syncwarp();
    } else if (warp >= 4) {
        const int bt = threadIdx.x - 128;
        int s = (kb1 - kb0) % p.stages;
        uint32_t ph = (uint32_t)((kb1 - kb0) / p.stages) & 1u;
        int id[1] = {adapter_of_warp_row(p.rows, bt & ~31, lane)}, slot[1];
        const int used = ap_find(sh.find, sh.list, id, slot, bt);
        const int ext = used * p.Rp;
        sh.slot[bt] = slot[0];
        if (bt == 0) sh.ext = ext;
        builders_sync();
        mbar_arrive(&sh.ifull);
        const __nv_bfloat16* trow = p.t + (size_t)bt * p.t_terms * p.Rp;
        const int cpr = ROWS ? p.nt >> 3 : 4, cj = bt % cpr, row0 = bt / cpr, step = 128 / cpr;
        const bool row_there = (uint32_t)bt * 128u < p.a_bytes;
        bool waited = false, ok = true;
        if (TERMS == 3 && early > 0) {
            const int q = warp & 3, row = q * 32 + lane;
            float4* const to = reinterpret_cast<float4*>(ap_raw + (ring - smem_u32(ap_raw)) + p.early + (size_t)row * pitch * 4);
#pragma unroll 1
            for (int c = 0, acc = 0, use = 0; c < early; ++c) {
                if (!__all_sync(0xffffffffu, mbar_wait(&sh.cfull[acc], (uint32_t)use & 1, abort_flag))) { give_up(100); ok = false; break; }
                tc_fence_after();
                if (q * 32 < p.rows.M) {
#pragma unroll 1
                    for (int col = 0; col < p.nt; col += 16) {
                        uint32_t v[16];
                        tmem_ld_x16(tmem + (uint32_t)acc * p.acc_cols + ((uint32_t)(q * 32) << 16) + col, v);
                        tmem_ld_wait();
                        if (row < p.rows.M) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                float4 x = c ? to[col / 4 + i] : make_float4(0.f, 0.f, 0.f, 0.f);
                                x.x += __uint_as_float(v[4 * i]); x.y += __uint_as_float(v[4 * i + 1]); x.z += __uint_as_float(v[4 * i + 2]); x.w += __uint_as_float(v[4 * i + 3]);
                                to[col / 4 + i] = x;
                            }
                        }
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.cempty[acc]);
                if (++acc == p.accs) { acc = 0; ++use; }
            }
            ok = !builders_any(!ok);
        }
        uint4 fv[8];
        auto load_f = [&](int e0) { ap_load_f<Kind>(p, sh.list, e0, min(WIDTH, ext - e0), p.nt, row0, step, cj, [&](int i) { return c0 + i; }, fv); };
        if (ok && rank * WIDTH < ext) load_f(rank * WIDTH);                    // f needs no waiting, t is the kernel's in front
#pragma unroll 1
        for (int e0 = rank * WIDTH; e0 < ext && ok; e0 += p.split * WIDTH) {
            uint4 tv[WIDTH / 8][TERMS];
            const int w = min(WIDTH, ext - e0);
            if (!waited) {
                grid_dependency_wait();
                waited = true;
                if (p.cache && row_there) {                    // the row's T at hand for all of its blocks
                    uint4* const to = reinterpret_cast<uint4*>(cache + (size_t)bt * p.t_terms * p.Rp);
                    if (slot[0] >= 0)
                        for (int i = 0; i < p.t_terms * p.Rp / 8; ++i) to[i] = __ldcg(reinterpret_cast<const uint4*>(trow) + i);
                    trow = cache + (size_t)bt * p.t_terms * p.Rp;
                }
            }
            ap_load_t<Kind>(trow, slot[0], p.Rp, e0, w, tv);
            if (any_odd(fv)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) fv[i] = make_uint4(finite_halves(fv[i].x), finite_halves(fv[i].y), finite_halves(fv[i].z), finite_halves(fv[i].w));
                for (int k = 0; k < p.split; ++k)
                    asm volatile("red.relaxed.cluster.shared::cluster.max.s32 [%0], %1;" ::"r"(p.split > 1 ? mapa_shared(smem_u32(&sh.odd), k) : smem_u32(&sh.odd)), "r"(1) : "memory");
            }
            const bool slot_free = __all_sync(0xffffffffu, mbar_wait(&sh.loads, 0, abort_flag) && mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag));
            if (!slot_free) give_up(96);
            if (slot_free) {
                const uint32_t a = ring + (uint32_t)s * p.stage_bytes;
                ap_store_block<Kind>(a, a + p.a_bytes, bt, row_there, w, p.nt, row0, step, cj, fv, tv);
            }
            fence_proxy_async_smem();
            if (builders_any(!slot_free)) { ok = false; break; }
            if (bt == 0) mbar_arrive(&sh.full[s]);
            if (++s == p.stages) { s = 0; ph ^= 1; }
            if (e0 + p.split * WIDTH < ext) load_f(e0 + p.split * WIDTH);
        }
        if (!waited) grid_dependency_wait();
    }
    if (warp == 2 && (p.flags & DR_BIAS)) {
        const int width = p.nt / p.split;
        for (int i = lane; i < width; i += 32) sh.bias[i] = c0 + rank * width + i < p.C ? __ldg(p.bias + c0 + rank * width + i) : 0.f;
    }
    // the adapters' f on its way to L2 while t is still being made: the cluster's CTAs share the list
    if (warp == 3) {
        if (!__all_sync(0xffffffffu, mbar_wait(&sh.ifull, 0, abort_flag))) {
            give_up(98);
        } else {
            const int used = sh.ext / p.Rp, cols = min(p.nt, p.C - c0), pieces = ROWS ? p.R * ((cols + 63) >> 6) : (cols * p.R + 63) >> 6;       // lines of 128 bytes
            for (int d = rank; d < used; d += p.split)
                for (int i = lane; i < pieces; i += 32) {
                    const __nv_bfloat16* at = ROWS ? p.f + ((size_t)sh.list[d] * p.R + i % p.R) * p.ldf + c0 + 64 * (i / p.R) : p.f + ((size_t)sh.list[d] * p.C + c0) * p.R + 64 * i;
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(at));
                }
        }
    }
    // the accumulators' rows into shared memory
    if (warp >= 4) {
        const int q = warp & 3, row = q * 32 + lane;
        if (q * 32 < p.rows.M) {
            if (!__all_sync(0xffffffffu, mbar_wait(&sh.tfull, 0, abort_flag))) {
                give_up(97);
            } else {
                tc_fence_after();
                const int ext = sh.ext;
                const bool own = ext > rank * WIDTH;             // this CTA had a further block
#pragma unroll 1
                for (int c = 0; c < p.nt; c += 32) {
#pragma unroll 1
                    for (int k = 0; k < (DUAL ? 2 : 1); ++k) {
                        uint32_t v[32];
                        tmem_ld_x32(tmem + (uint32_t)k * p.acc_cols + ((uint32_t)(q * 32) << 16) + c, v);
                        tmem_ld_wait();
                        if (TERMS == 3) {
#pragma unroll 1
                            for (int a = 1; a < min(chains, p.accs); ++a) {
                                uint32_t w[32];
                                tmem_ld_x32(tmem + (uint32_t)a * p.acc_cols + ((uint32_t)(q * 32) << 16) + c, w);
                                tmem_ld_wait();
#pragma unroll
                                for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(w[i]));
                            }
                            if (early > 0 && row < p.rows.M) {
                                const float4* from = reinterpret_cast<const float4*>(ap_raw + (ring - smem_u32(ap_raw)) + p.early + (size_t)row * pitch * 4 + c * 4);
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    if (c + 4 * i >= p.nt) break;
                                    const float4 x = from[i];
                                    v[4 * i] = __float_as_uint(__uint_as_float(v[4 * i]) + x.x);
                                    v[4 * i + 1] = __float_as_uint(__uint_as_float(v[4 * i + 1]) + x.y);
                                    v[4 * i + 2] = __float_as_uint(__uint_as_float(v[4 * i + 2]) + x.z);
                                    v[4 * i + 3] = __float_as_uint(__uint_as_float(v[4 * i + 3]) + x.w);
                                }
                            }
                        }
                        if (row < p.rows.M) {
                            float4* to = reinterpret_cast<float4*>(sums + ((size_t)k * p.rows.M + row) * pitch + c);
                            const bool there = k == 0 || own;
#pragma unroll
                            for (int i = 0; i < 8; ++i)
                                if (c + 4 * i < p.nt)
                                    to[i] = there ? make_float4(__uint_as_float(v[4 * i]), __uint_as_float(v[4 * i + 1]), __uint_as_float(v[4 * i + 2]), __uint_as_float(v[4 * i + 3]))
                                                  : make_float4(0.f, 0.f, 0.f, 0.f);
                        }
                    }
                }
            }
        }
    }
    tc_fence_before();
    ap_settle(abort_flag);
    if (p.split > 1) cluster_sync_all();
    {
        const int width = p.nt / p.split, quads = width >> 2;
        const bool odd = sh.odd != 0;
        const float low = (p.flags & DR_RELU) ? 0.f : -INFINITY;
        for (int i = threadIdx.x; i < p.rows.M * quads; i += AP_FEW_THREADS) {
            const int m = i / quads, cl = rank * width + 4 * (i - m * quads), c = c0 + cl;
            const int slot = sh.slot[m];
            if (slot == ROW_NONE || c >= p.C) continue;
            const uint32_t at = smem_u32(sums + (size_t)m * pitch + cl), at2 = smem_u32(sums + ((size_t)p.rows.M + m) * pitch + cl);
            float v[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
            auto gather = [&](uint32_t from, float (&to)[4]) {
                float4 x[8];                                   // all on their way before the first is added
#pragma unroll
                for (int k = 0; k < 8; ++k) if (k < p.split) x[k] = ld_shared_cluster_f4(p.split > 1 ? mapa_shared(from, (uint32_t)k) : from);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < p.split) { to[0] += x[k].x; to[1] += x[k].y; to[2] += x[k].z; to[3] += x[k].w; }
            };
            gather(at, v);
            if (DUAL) gather(at2, u);
            const uint32_t bits = DUAL ? __ldcg(p.mask + (size_t)m * p.ldm + (c >> 5)) >> (c & 31) : 0xFu;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (DUAL && (bits >> k & 1)) v[k] += u[k];
                if (odd && slot >= 0 && c + k < p.C && (bits >> k & 1)) v[k] += ap_odd<ROWS>(p, sh.list[slot], m, c + k);
                if (p.flags & DR_BIAS) v[k] += sh.bias[cl - rank * width + k];
                v[k] = max_nan(v[k], low);
            }
            const size_t to = (size_t)m * p.ldo + c;
            if (p.out_vec && c + 4 <= p.C) {
                if (TERMS == 3) *reinterpret_cast<float4*>((float*)p.out + to) = make_float4(v[0], v[1], v[2], v[3]);
                else *reinterpret_cast<uint2*>((__nv_bfloat16*)p.out + to) = make_uint2(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (c + k < p.C) {
                        if (TERMS == 3) ((float*)p.out)[to + k] = v[k];
                        else ((__nv_bfloat16*)p.out)[to + k] = __float2bfloat16_rn(v[k]);
                    }
            }
        }
    }
    __syncthreads();
    if (p.split > 1) cluster_sync_all();                       // no CTA leaves while another reads its sums
    if (warp == 1) tmem_dealloc(tmem, p.tmem_cols);
}

static int ap_map(CUtensorMap* map, const void* ptr, size_t rows, size_t inner, size_t ld, int box_inner, int box_rows) {
    const cuuint64_t dims[2] = {inner, rows}, strides[1] = {ld * 2};
    const cuuint32_t box[2] = {(cuuint32_t)box_inner, (cuuint32_t)box_rows};
    return tmap_tiled(map, 2, ptr, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

template <class Kernel, class... Args>
static int ap_start(Kernel k, PerDeviceFlag& ready, int grid, int threads, int cluster, bool overlap, size_t smem, cudaStream_t s, const Args&... args) {
    if (!ready.get()) {
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, AP_SMEM_MOST) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
        ready.set();
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)cluster; attr[n].val.clusterDim.y = 1; attr[n].val.clusterDim.z = 1;
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
template <class Kind>
static int ap_launch(const CUtensorMap& mz, const CUtensorMap& mw, const CUtensorMap& mo, const ApParams& p, bool overlap, size_t smem, cudaStream_t s) {
    static PerDeviceFlag ready;
    const int units = Kind::PAIR ? num_sms() / 2 : num_sms();
    return ap_start(adapter_product_kernel<Kind>, ready, std::min(p.tiles, units) * (Kind::PAIR ? 2 : 1), AP_THREADS, Kind::PAIR ? 2 : 1, overlap, smem, s, mz, mw, mo, p);
}
template <class Kind>
static int ap_launch_few(const CUtensorMap& mz, const CUtensorMap& mw, const ApParams& p, bool overlap, size_t smem, cudaStream_t s) {
    static PerDeviceFlag ready;
    return ap_start(adapter_few_kernel<Kind>, ready, p.tiles_c * p.split, AP_FEW_THREADS, p.split, overlap, smem, s, mz, mw, p);
}

// Clusters of so many CTAs that the device holds at a time (a cluster lies within a group of SMs, so they are fewer than the SMs suggest).
static int few_clusters(int ctas) {
    static std::atomic<int> known[4][64];
    const int d = PerDeviceFlag::dev(), i = ctas == 1 ? 0 : ctas == 2 ? 1 : ctas == 4 ? 2 : 3;
    if (i == 0) return num_sms();
    int n = known[i][d].load(std::memory_order_relaxed);
    if (n == 0) {
        auto* k = adapter_few_kernel<ApKind<false, false, false, false, 2>>;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(num_sms() / ctas * ctas));
        cfg.blockDim = dim3(AP_FEW_THREADS);
        cfg.dynamicSmemBytes = AP_SMEM;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, AP_SMEM_MOST) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, k, &cfg) != cudaSuccess || n < 1) {
            (void)cudaGetLastError();
            n = num_sms() / (2 * ctas);
        }
        known[i][d].store(n, std::memory_order_relaxed);
    }
    return n;
}

static int few_run(const ProductArgs& a, ApParams& p, bool overlap, cudaStream_t s) {
    const int M = a.rows.M, sms = num_sms();
    const bool dual = a.mask;
    p.a_bytes = (uint32_t)((M + 7) / 8 * 8) * 128u;
    // Width of a tile and CTAs that share its l, by a model in cycles: w once from memory (3.4 KB a cycle for all SMs), a CTA's loads at 32 bytes a
    // cycle and 150 cycles a stage, 1500 for the meeting of a cluster.  For 32 x 4096 x 4096 it picks 128 columns and four CTAs, 24.6 us; measured when
    // that took 27, 64 and two took 33, 32 alone 50, 128 alone 57.
    double best = 0.;
    const bool f32 = a.flags & DR_OUT_F32;
    for (int nt = a.transposed ? 64 : 16; nt <= (f32 ? 64 : 128); nt *= 2)
        for (int split = 1; split <= 8 && split <= p.kblocks && 4 * split <= nt; split *= 2) {
            const int tiles = (a.C + nt - 1) / nt, blocks = (p.kblocks + split - 1) / split;
            const int waves = (tiles + few_clusters(split) - 1) / few_clusters(split);
            const double cta = blocks * ((p.a_bytes + nt * 128.) / 32. + 150.);
            const double t = std::max(waves * cta, (double)a.C * a.L * 2. / 3400.) + (split > 1 ? 1500. : 0.) + waves * 2. * nt;
            if (best == 0. || t < best) { best = t; p.nt = nt; p.split = split; }
        }
    p.tiles_c = (a.C + p.nt - 1) / p.nt;
    p.tiles = p.tiles_c;
    p.b_bytes = (uint32_t)p.nt * 128u;
    p.stage_bytes = p.a_bytes + p.b_bytes;
    p.acc_cols = std::max(32, p.nt);
    const int blocks = (p.kblocks + p.split - 1) / p.split;                   // of a CTA, at most
    p.accs = f32 ? std::min(256 / (int)p.acc_cols, blocks / AP_CHAIN + 1) : 1;
    p.tmem_cols = p.acc_cols * (dual ? 2 : 1);
    while (p.tmem_cols < p.acc_cols * p.accs) p.tmem_cols *= 2;
    const size_t sums = (size_t)M * (p.nt + 4) * 4 * (dual ? 2 : 1), early = f32 && blocks > p.accs * AP_CHAIN ? sums : 0;
    const uint32_t slack = 16384u - p.a_bytes;                                // the MMA reads 128 rows from the last stage on
    p.stages = (int)std::min<uint32_t>(AP_MAX_STAGES, (std::min<uint32_t>(AP_SMEM, AP_SMEM_MOST - 1024 - (uint32_t)early) - slack) / p.stage_bytes);
    const size_t ring = (size_t)p.stages * p.stage_bytes + slack;
    const size_t rows_t = (size_t)(M + 7) / 8 * 8 * a.terms * a.Rp * 2, behind = std::max(ring, sums) + early;
    p.early = (int)(behind - early);
    p.cache = behind + rows_t <= AP_SMEM_MOST - 1024 ? (int)behind : 0;
    const size_t smem = std::max<size_t>(AP_FEW_SMEM, 1024 + behind + (p.cache ? rows_t : 0));
    alignas(64) CUtensorMap mz, mw;
    int rc = ap_map(&mz, a.z, M, a.L, a.ldz, 64, (M + 7) / 8 * 8);
    if (rc != DR_OK) return rc;
    rc = a.transposed ? ap_map(&mw, a.w, a.L, a.C, a.ldw, 64, 64) : ap_map(&mw, a.w, a.C, a.L, a.ldw, 64, p.nt);
    if (rc != DR_OK) return rc;
    if (a.transposed) return dual ? ap_launch_few<ApKind<false, false, true, true, 2>>(mz, mw, p, overlap, smem, s) : ap_launch_few<ApKind<false, false, true, false, 2>>(mz, mw, p, overlap, smem, s);
    return (a.flags & DR_OUT_F32) ? ap_launch_few<ApKind<false, false, false, false, 3>>(mz, mw, p, overlap, smem, s) : ap_launch_few<ApKind<false, false, false, false, 2>>(mz, mw, p, overlap, smem, s);
}

int adapter_product_run(const ProductArgs& a, bool overlap, cudaStream_t s) {
    ApParams p = {};
    p.rows = a.rows;
    p.L = a.L; p.C = a.C; p.R = a.R; p.Rp = a.Rp;
    p.rp_magic = (uint32_t)((0x100000000ull + a.Rp - 1) / a.Rp);
    p.row_id = a.row_id; p.t = a.t; p.t_terms = a.terms; p.bias = a.bias; p.f = a.f; p.ldf = a.ldf;
    p.f_vec = !a.transposed && (a.R & 7) == 0;
    p.flags = a.flags; p.out = a.out; p.ldo = a.ldo; p.mask = a.mask; p.ldm = a.ldm;
    const bool dual = a.mask, f32 = a.flags & DR_OUT_F32;
    const size_t size = f32 ? 4 : 2;
    p.out_vec = aligned16(a.out) && (a.ldo * size) % 16 == 0;
    p.status = dev_status_ptr();
    p.kblocks = (a.L + 63) / 64;
    const int M = a.rows.M, sms = num_sms();
    if (M <= AP_TILE) return few_run(a, p, overlap, s);
    const long long rows128 = (M + 127) / 128;
    const int gran = a.transposed ? 64 : 16;
    // Tile: as wide as leaves every SM one, by pairs where the pairs have enough tiles
    const int most = dual || f32 ? 128 : 256;
    bool pair = false, wide = false;
    int nt = std::min(most, (a.C + gran - 1) / gran * gran);
    if (rows128 * ((a.C + nt - 1) / nt) < sms) {
        const long long want = std::max(1ll, sms / rows128);         // column blocks that give every SM a tile
        nt = (int)((a.C + want - 1) / want);
        nt = std::min(most, std::max(gran, (nt + gran - 1) / gran * gran));
    } else if (a.C >= 128 && a.L >= 512 && !dual) {
        // A pair reads less of w, but its rows are of more adapters, and behind a mask its drains bound it: 12544 x 2048 x 64 alone 38 us, by pairs 42;
        // x 512 54 and 52; x 2048 124 and 110; with images of 49 rows x 512 65 and 71 (l alone
        // does not tell, and the rule takes the pair there); behind a mask x 512 91 and 107, x 2048 181 and 196
        const int pn = a.C > 128 ? most : 128;
        const long long pairs = ((rows128 + 1) / 2) * ((a.C + pn - 1) / pn);
        if (pairs >= sms / 2) { pair = true; nt = pn; }
        // Out of L2 a pair's block of 256 x 256 takes 64 KB for 512 cycles of MMAs, more than the 12 TB/s that all SMs get; 256 x 512 takes 96 KB
        // for 1024, but its accumulators fill the tensor memory, so a tile's drain is only half hidden: long l.  16384 x 4096 x 4096 takes 370 us
        // instead of 509.
        if (pair && !f32 && a.L >= 1024 && a.C >= 512 && ((rows128 + 1) / 2) * ((a.C + 511) / 512) >= sms / 2) { wide = true; nt = 512; }
    }
    p.nt = nt;
    p.tiles_c = (a.C + nt - 1) / nt;
    const long long tiles = (pair ? (rows128 + 1) / 2 : rows128) * p.tiles_c;
    if (tiles > 0x7fffffffll) return DR_ERR_UNSUPPORTED;
    p.tiles = (int)tiles;
    const int cols = pair ? nt / 2 : nt;
    p.a_bytes = AP_TILE * 128u;
    p.b_bytes = (uint32_t)cols * 128u;
    p.stage_bytes = p.a_bytes + p.b_bytes;
    p.stages = (int)std::min<uint32_t>(AP_MAX_STAGES, AP_SMEM / p.stage_bytes);
    p.acc_cols = f32 ? 32 : 64;             // the drain reads 128 bytes of results at a time, whatever the tile's width
    while ((int)p.acc_cols < (wide ? 256 : nt)) p.acc_cols *= 2;
    p.tmem_cols = p.acc_cols * (dual ? 4 : 2);
    const size_t smem = 1024 + (size_t)p.stages * p.stage_bytes + 8 * 4096;
    alignas(64) CUtensorMap mz, mw, mo = {};
    int rc = ap_map(&mz, a.z, M, a.L, a.ldz, 64, AP_TILE);
    if (rc != DR_OK) return rc;
    rc = a.transposed ? ap_map(&mw, a.w, a.L, a.C, a.ldw, 64, 64) : ap_map(&mw, a.w, a.C, a.L, a.ldw, 64, wide ? 128 : cols);
    if (rc == DR_OK && p.out_vec) rc = ap_map(&mo, a.out, M, (size_t)a.C * (f32 ? 2 : 1), a.ldo * (f32 ? 2 : 1), 64, 32);
    if (rc != DR_OK) return rc;
    //                                     PAIR  WIDE   ROWS  DUAL TERMS
    if (a.transposed) {
        if (wide) return ap_launch<ApKind<true, true, true, false, 2>>(mz, mw, mo, p, overlap, smem, s);
        if (pair) return ap_launch<ApKind<true, false, true, false, 2>>(mz, mw, mo, p, overlap, smem, s);
        return dual ? ap_launch<ApKind<false, false, true, true, 2>>(mz, mw, mo, p, overlap, smem, s) : ap_launch<ApKind<false, false, true, false, 2>>(mz, mw, mo, p, overlap, smem, s);
    }
    if (wide) return ap_launch<ApKind<true, true, false, false, 2>>(mz, mw, mo, p, overlap, smem, s);
    if (pair) return f32 ? ap_launch<ApKind<true, false, false, false, 3>>(mz, mw, mo, p, overlap, smem, s) : ap_launch<ApKind<true, false, false, false, 2>>(mz, mw, mo, p, overlap, smem, s);
    return f32 ? ap_launch<ApKind<false, false, false, false, 3>>(mz, mw, mo, p, overlap, smem, s) : ap_launch<ApKind<false, false, false, false, 2>>(mz, mw, mo, p, overlap, smem, s);
}

}  // namespace dr
