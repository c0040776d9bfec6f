// The adapters' first product, out[m][r] = factor * sum_l D(z)[m][l] f_a[r][l] with a the adapter of row m: few columns, so it is bound
// by the bytes of z (and, for single rows, of f).  Warps multiply fragments (mma.sync) that they load straight from memory: the order of l
// within a product is free, so a thread takes 16 consecutive l of its rows with 16-byte loads and its values of four MMAs lie in its own
// registers; no shared memory, and the dropout's mask is drawn where the values are.  A warp whose rows belong to several adapters does
// the product once for each and keeps the rows that are that adapter's.  200704 x 64, rank 8, behind a dropout: 21 us, half of it the generator; 32 x 4096,
// rank 16, 32 adapters: 7 us, all latency.
//
// Few rows: the warps of a CTA share 16 rows and split l, a cluster of CTAs takes ranges of l (their sums meet in distributed shared memory, in
// order), and further clusters take adapters of their own.
//
// The tensor cores cut their sums off instead of rounding them, about 1.5e-8 of the result for each product of 16 l in a row, so 512 l are summed at a time
// and those sums added up in float32.  Fragments (LONG, where a warp has more l than that): in shared memory, a place for each of a thread's sums, since
// registers for them would halve the warps of an SM.  In one sum t of 40000 x 9216 was off by 1.0e-5, and is by 5e-7; 437 us, and 440 with the adding up,
// up to 4 % more for other sizes.
#include <algorithm>

#include "adapter.cuh"
#include "conv_common.cuh"
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

constexpr int DOWN_CHAIN = 8;                          // blocks of 64 l

// MT tiles of 16 rows, RT tiles of 8 columns a warp; JOIN: the 8 warps of a CTA split l over the same rows, else each has rows of its own
// Few rows: 64 registers, so that the next kernel's CTAs (32768 registers each) find room beside two of these.  LONG: what two CTAs an SM leave, where the
// sums without a generator fit that (20000 x 9216, rank 32: 202 us, with 132 registers 262)
template <int MT, int RT, bool DROP, bool JOIN, bool LONG>
__global__ void __launch_bounds__(256, LONG ? (RT <= 4 && !DROP ? 2 : 0) : MT == 1 && RT <= 2 && !DROP ? 4 : 0) adapter_down_kernel(const DownParams p) {
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
    ptx::grid_dependency_wait();                                 // f may be the work of the kernel in front

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
        // columns behind the rank are zeros whatever the row or the scale holds: 0 * inf would be NaN in the whole row of the second product
        split3(r < p.R ? x * scale : 0.f, r + 1 < p.R ? y * scale : 0.f, u[0], u[1], u[2]);
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
        extern __shared__ float down_sums[];                     // LONG: [MT * RT * 4][256]
        float* const sums = down_sums + threadIdx.x;
        int left = DOWN_CHAIN;
        bool summed = false;
        auto add_sums = [&]() {
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int r = 0; r < RT; ++r)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[t][r][i] += sums[((t * RT + r) * 4 + i) * 256];
        };
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
            if (LONG && --left == 0) {
                if (summed) add_sums();
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int r = 0; r < RT; ++r)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            sums[((t * RT + r) * 4 + i) * 256] = acc[t][r][i];
                            acc[t][r][i] = 0.f;
                        }
                summed = true;
                left = DOWN_CHAIN;
            }
        }
        if (LONG && summed) add_sums();
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
                        float x = 0.f, y = 0.f, u[8], v[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k)               // all on their way before the first is added
                            if (k < p.ks)
                                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(u[k]), "=f"(v[k]) : "r"(ptx::mapa_shared(ptx::smem_u32(range + row * RT * 8 + r), (uint32_t)k)) : "memory");
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (k < p.ks) { x += u[k]; y += v[k]; }
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

// ---- many rows, long l, ranks over 16, requests of many rows --------------------------------------------------------------------------------
// The same product on tcgen05: a CTA takes 128 rows, z and the adapter's rows come by TMA into a ring, the accumulator (128 x rank) lies in TMEM.  Rows
// of several adapters: the product is run once for each.  512 l are summed at a time and the drain adds those up in float32 (all 4096 at once: 5e-6 of a
// gradient built on them, so 9e-7).  16384 x 4096, rank 64: 35 us, with fragments
// from memory 82 (every 32 rows read all of an adapter).
constexpr int DT_THREADS = 192, DT_STAGES = 4;         // warp 0 loads, 1 issues MMAs, 2-5 find the adapters and drain; two CTAs to an SM
constexpr int DT_CHAIN = 8;                            // blocks of 64 l

struct DownTileParams {
    AdRows rows;
    int L, R, Rp, n, kblocks, terms;
    float factor, after;
    const float* scale;
    __nv_bfloat16* out;
    float* keep;
    int* row_id;
    int* status;
};
struct DownTileShared {
    uint64_t full[DT_STAGES], empty[DT_STAGES], tfull[2], tempty[2], found;
    uint32_t tmem;
    int abort, used;
    uint16_t list[128];
    ApFind find;
};

__global__ void __launch_bounds__(DT_THREADS, 2)
adapter_down_tile_kernel(const __grid_constant__ CUtensorMap map_z, const __grid_constant__ CUtensorMap map_f, const __grid_constant__ DownTileParams p) {
    using namespace ptx;
    extern __shared__ uint8_t dt_raw[];
    __shared__ DownTileShared sh;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const uint32_t ring = (smem_u32(dt_raw) + 1023u) & ~1023u;
    const uint32_t stage_bytes = 16384u + (uint32_t)p.n * 128u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, m0 = (int)blockIdx.x * 128, r0 = (int)blockIdx.y * 64;
    volatile int* abort_flag = &sh.abort;
    if (threadIdx.x == 0) {
        for (int i = 0; i < DT_STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], 1); mbar_init(&sh.tempty[i], 4); }
        mbar_init(&sh.found, 128);
        sh.abort = 0;
        fence_barrier_init();
        prefetch_tensormap(&map_z);
        prefetch_tensormap(&map_f);
    }
    if (warp == 1) { tmem_alloc(&sh.tmem, 128); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem, full0 = smem_u32(&sh.full[0]), empty0 = smem_u32(&sh.empty[0]);
    auto give_up = [&](int site) {
        if (!*abort_flag) report_timeout(p.status, site, (int)blockIdx.x);
        *abort_flag = 1;
    };
    if (warp == 0) {
        if (lane == 0) {
            grid_dependency_wait();                              // f may be the work of the kernel in front
            if (!mbar_wait(&sh.found, 0, abort_flag)) {
                give_up(111);
            } else {
                int s = 0;
                uint32_t ph = 0;
                bool ok = true;
                for (int d = 0; d < sh.used && ok; ++d) {
                    const int row = sh.list[d] * p.R + r0;
                    for (int kb = 0; kb < p.kblocks; ++kb) {
                        if (!mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag)) { give_up(112); ok = false; break; }
                        const uint32_t a = ring + (uint32_t)s * stage_bytes, bar = full0 + 8 * s;
                        mbar_expect_tx_u32(bar, stage_bytes);
                        tma_load_2d_u32<false>(a, &map_z, bar, kb << 6, m0, 1u);
                        tma_load_2d_u32<false>(a + 16384u, &map_f, bar, kb << 6, row, 1u);
                        if (++s == DT_STAGES) { s = 0; ph ^= 1; }
                    }
                }
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            if (!mbar_wait(&sh.found, 0, abort_flag)) {
                give_up(113);
            } else {
                const uint32_t idesc = make_idesc_bf16(128, p.n);
                const int tail16 = ((p.L - ((p.kblocks - 1) << 6)) + 15) >> 4;
                int s = 0;
                uint32_t ph = 0;
                bool ok = true;
                for (int d = 0, n = 0; d < sh.used && ok; ++d) {
                    for (int k0 = 0; k0 < p.kblocks && ok; k0 += DT_CHAIN, ++n) {
                        if (!mbar_wait(&sh.tempty[n & 1], (uint32_t)((n >> 1) & 1) ^ 1, abort_flag)) { give_up(114); ok = false; break; }
                        tc_fence_after();
                        for (int kb = k0; kb < min(p.kblocks, k0 + DT_CHAIN); ++kb) {
                            if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(115); ok = false; break; }
                            tc_fence_after();
                            const uint32_t a = sdesc_lo(ring + (uint32_t)s * stage_bytes), b = sdesc_lo(ring + (uint32_t)s * stage_bytes + 16384u);
                            const int n16 = kb == p.kblocks - 1 ? tail16 : 4;
#pragma unroll
                            for (int k = 0; k < 4; ++k) umma_bf16_lo<false>(tmem + 64u * (n & 1), a + 2 * k, b + 2 * k, idesc, kb > k0 || k ? 1u : 0u, k < n16 ? 1u : 0u);
                            umma_commit_u32<false>(empty0 + 8 * s);
                            if (++s == DT_STAGES) { s = 0; ph ^= 1; }
                        }
                        umma_commit(&sh.tfull[n & 1]);
                    }
                }
            }
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- a thread to a row: TMEM lanes 32 (warp mod 4) + lane
        const int q = warp & 3, row = 32 * q + lane, m = m0 + row;
        int id[1] = {adapter_of_warp_row(p.rows, m0 + 32 * q, lane)}, slot[1];
        if (m < p.rows.M && p.row_id && r0 == 0) p.row_id[m] = id[0];
        const int used = ap_find(sh.find, sh.list, id, slot, (int)threadIdx.x - 64);
        if (threadIdx.x == 64) sh.used = used;
        builders_sync();
        mbar_arrive(&sh.found);
        const float scale = (id[0] >= 0 && p.scale ? __ldg(p.scale + id[0]) : 1.f) * p.after;
        const int rn = min(64, p.Rp - r0);
        if (p.keep && id[0] == ROW_SHARED)
            for (int r = r0; r < min(p.R, r0 + 64); ++r) p.keep[(size_t)m * p.R + r] = 0.f;
        float sum[8][8];
        bool ok = true;
        for (int d = 0, n = 0; d < used && ok; ++d) {
#pragma unroll
            for (int b = 0; b < 8; ++b)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[b][i] = 0.f;
            for (int k0 = 0; k0 < p.kblocks; k0 += DT_CHAIN, ++n) {
                if (!__all_sync(0xffffffffu, mbar_wait(&sh.tfull[n & 1], (uint32_t)(n >> 1) & 1, abort_flag))) { give_up(116); ok = false; break; }
                tc_fence_after();
#pragma unroll
                for (int b = 0; b < 8; ++b) {
                    if (8 * b >= rn) break;
                    uint32_t v[8];
                    tmem_ld_x8(tmem + 64u * (n & 1) + 8 * b + ((uint32_t)(q * 32) << 16), v);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i) sum[b][i] += __uint_as_float(v[i]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.tempty[n & 1]);
            }
            if (!ok || slot[0] != d) continue;
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const int r = r0 + 8 * b;
                if (8 * b >= rn) break;
                float t[8], ts[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    t[i] = sum[b][i] * p.factor;
                    ts[i] = r + i < p.R ? t[i] * scale : 0.f;                  // columns behind the rank are the next adapter's
                }
                if (p.keep) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) if (r + i < p.R) p.keep[(size_t)m * p.R + r + i] = t[i];
                }
                uint32_t u[3][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) split3(ts[2 * i], ts[2 * i + 1], u[0][i], u[1][i], u[2][i]);
                __nv_bfloat16* to = p.out + (size_t)m * p.terms * p.Rp + r;
#pragma unroll
                for (int k = 0; k < 3; ++k)
                    if (k < p.terms) *reinterpret_cast<uint4*>(to + (size_t)k * p.Rp) = make_uint4(u[k][0], u[k][1], u[k][2], u[k][3]);
            }
        }
    }
    tc_fence_before();
    ap_settle(abort_flag);
    if (warp == 1) tmem_dealloc(tmem, 128);
}

static int down_tile_run(const AdRows& rows, int L, int R, int Rp, const __nv_bfloat16* z, size_t ldz, const __nv_bfloat16* f, size_t ldf, float factor,
                         const float* scale, float after, int terms, __nv_bfloat16* out, float* keep, int* row_id, bool overlap, cudaStream_t s) {
    DownTileParams p = {rows, L, R, Rp, R >= 64 ? 64 : (R + 15) / 16 * 16, (L + 63) / 64, terms, factor, after, scale, out, keep, row_id, dev_status_ptr()};
    alignas(64) CUtensorMap mz, mf;
    auto map = [](CUtensorMap* m, const void* ptr, size_t n, int cols, size_t ld, int box_rows) {
        const cuuint64_t dims[2] = {(cuuint64_t)cols, n}, strides[1] = {ld * 2};
        const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
        return tmap_tiled(m, 2, ptr, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
    };
    int rc = map(&mz, z, rows.M, L, ldz, 128);
    if (rc == DR_OK) rc = map(&mf, f, (size_t)rows.adapters * R, L, ldf, p.n);
    if (rc != DR_OK) return rc;
    const int smem = 1024 + DT_STAGES * (16384 + p.n * 128);
    static PerDeviceFlag ready;
    if (!ready.get()) {
        if (cudaFuncSetAttribute(adapter_down_tile_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 1024 + DT_STAGES * (16384 + 64 * 128)) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
        ready.set();
    }
    return start_kernel(adapter_down_tile_kernel, dim3((unsigned)((rows.M + 127) / 128), (unsigned)((R + 63) / 64)), DT_THREADS, 1, overlap, smem, s, mz, mf, p);
}

DownPlan adapter_down_plan(int M, int L, int R, int adapters, int segments, bool dropped) {
    DownPlan d = {};
    // Tiles of 128 rows nearly for every SM, of mostly one adapter each, and enough l and columns that a tile's start does not show
    d.tile = !dropped && M >= 96 * num_sms() && M >= 128ll * segments && L >= 512 && R > 16;
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

template <int MT, int RT, bool JOIN, bool LONG>
static int down_launch(const DownPlan& d, const DownParams& p, bool overlap, cudaStream_t s) {
    const dim3 grid((unsigned)((p.rows.M + d.rows_cta - 1) / d.rows_cta), (unsigned)d.ks, (unsigned)(d.zsplit * d.rchunks));
    auto* const k = p.key.thr ? adapter_down_kernel<MT, RT, true, JOIN, LONG> : adapter_down_kernel<MT, RT, false, JOIN, LONG>;
    const int smem = LONG ? MT * RT * 4 * 256 * (int)sizeof(float) : 0;
    static PerDeviceFlag ready[2];
    const int i = p.key.thr ? 1 : 0;
    if ((MT == 1 || LONG) && !ready[i].get()) {
        // An SM changes how it divides its memory only when it is empty: with the largest part shared the next kernel's CTAs can begin beside this one's
        if (MT == 1 && cudaFuncSetAttribute(k, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
        if (LONG && cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
        ready[i].set();
    }
    return start_kernel(k, grid, 256, d.ks, overlap, smem, s, p);
}
template <int RT>
static int down_launch_rt(const DownPlan& d, const DownParams& p, bool overlap, cudaStream_t s) {
    const bool more = p.l_range > 64 * DOWN_CHAIN * d.warps_k;
    if (d.warps_k == 1) return more ? down_launch<2, RT, false, true>(d, p, overlap, s) : down_launch<2, RT, false, false>(d, p, overlap, s);
    if (d.mt == 2) return more ? down_launch<2, RT, true, true>(d, p, overlap, s) : down_launch<2, RT, true, false>(d, p, overlap, s);
    return more ? down_launch<1, RT, true, true>(d, p, overlap, s) : down_launch<1, RT, true, false>(d, p, overlap, s);
}

int adapter_down_run(const DownPlan& d, const AdRows& rows, int L, int R, int Rp, const __nv_bfloat16* z, size_t ldz, const __nv_bfloat16* f, size_t ldf,
                     const DropKey& key, float factor, const float* scale, float after, int terms, __nv_bfloat16* out, float* keep, int* row_id, bool overlap, cudaStream_t s) {
    if (d.tile) return down_tile_run(rows, L, R, Rp, z, ldz, f, ldf, factor, scale, after, terms, out, keep, row_id, overlap, s);
    DownParams p;
    p.rows = rows;
    p.L = L; p.L8 = (L + 7) / 8 * 8; p.R = R; p.Rp = Rp; p.ks = d.ks; p.zsplit = d.zsplit;
    p.l_range = (((L + d.ks - 1) / d.ks) + 63) / 64 * 64;
    p.z = z; p.f = f; p.ldz = ldz; p.ldf = ldf;
    p.key = key; p.factor = factor; p.scale = scale; p.after = after; p.terms = terms; p.out = out; p.keep = keep; p.row_id = row_id;
    if (d.rt == 1) return down_launch_rt<1>(d, p, overlap, s);
    if (d.rt == 2) return down_launch_rt<2>(d, p, overlap, s);
    return d.rt == 4 ? down_launch_rt<4>(d, p, overlap, s) : down_launch_rt<8>(d, p, overlap, s);
}

// ---- layouts ------------------------------------------------------------------------------------------------------
// Up to four tensors in one launch; a thread writes 16 bytes.
struct AlignJobs { AlignJob job[4]; };
__global__ void __launch_bounds__(256) adapter_align_kernel(const AlignJobs jobs) {
    const AlignJob& j = jobs.job[blockIdx.y];
    const size_t per = j.ldd >> 3, n = j.rows * per, stride = (size_t)gridDim.x * 256;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += stride) {
        const size_t row = i / per;
        const int c = 8 * (int)(i - row * per);
        const unsigned short* src = reinterpret_cast<const unsigned short*>(j.src) + row * j.ld + c;
        uint32_t u[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) u[k] = (c + 2 * k < j.cols ? (uint32_t)__ldg(src + 2 * k) : 0u) | (c + 2 * k + 1 < j.cols ? (uint32_t)__ldg(src + 2 * k + 1) << 16 : 0u);
        *reinterpret_cast<uint4*>(j.dst + row * j.ldd + c) = make_uint4(u[0], u[1], u[2], u[3]);
    }
}
int adapter_align_run(const AlignJob* jobs, int n, cudaStream_t s) {
    if (n == 0) return DR_OK;
    AlignJobs a = {};
    size_t most = 0;
    for (int i = 0; i < n; ++i) {
        a.job[i] = jobs[i];
        most = std::max(most, (jobs[i].rows * (jobs[i].ldd >> 3) + 255) / 256);
    }
    adapter_align_kernel<<<dim3((unsigned)std::min(most, (size_t)num_sms() * 16), (unsigned)n), 256, 0, s>>>(a);
    count_launch();
    return launch_status();
}

}  // namespace dr
