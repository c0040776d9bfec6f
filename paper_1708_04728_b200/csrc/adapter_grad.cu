// The adapters' gradients, g_a[r][c] = sum over the rows m of adapter a of P[m][r] D(z)[m][c]: with P = u and z = x the first factor's,
// with P = t and z = dy the second's.  Bound by the bytes of z: 16384 x 4096 and 4096, rank 64, in 75 us, 3.8 TB/s; 12544 x 2048 behind a dropout and 512, images of 49
// rows, in 28.
//
// The rows are sorted by adapter first (an index list; order within an adapter as in the tensor).  A CTA owns a column block and an even share of the
// sorted rows, whatever their adapters; where its share passes from one adapter to the next it writes what it has and starts over.  Share
// and adapter only grow along the list, so their sum numbers the partial results without gaps; they are added in order by a second
// kernel: the same result on every run, and no share is larger than another however the requests are spread.
//
// On the tensor cores (tcgen05): 128 columns of z are the rows of an accumulator in TMEM, P's columns its columns, so both operands have the contraction
// index m as their rows and are brought as they lie in memory by TMA, 128 bytes wide, into tiles of 64 rows in the 128-byte swizzle: 64 or 16
// rows that are neighbours in the tensor as one box, others gathered four at a time, with zeros for rows behind the last.  A thread takes about 100 cycles
// to issue one of these, whatever it brings (16384 x 4096 x 4096 with 112 gathers a stage 319 us, with 28 boxes 129), hence the larger boxes
// and three issuing warps.  P enters as three bfloat16 values, side by side, which the drain adds up.  With a
// dropout further warps clear the dropped values in place before the tile is multiplied, by a mask that is drawn once for all products that want it
// (12544 x 2048: the generator in this kernel cost 24 us and in that of dx 11, the one pass costs 13)
#include <algorithm>

#include "adapter.cuh"
#include "conv_common.cuh"
#include "umma_ptx.cuh"

namespace dr {
using namespace ptx;

// ---- what the backward pass lays out first, in one launch -------------------------------------------------------------------------------
struct PrepParams {
    AdRows rows;
    int sort_blocks, turn_x, turn_y, turn_blocks, term_blocks;
    int *perm, *start;
    int N, R, Rp;
    const __nv_bfloat16* b;     // [adapters][N][R], turned to bt [adapters][R][ldb]
    __nv_bfloat16* bt;
    size_t ldb;
    const float *t, *scale;     // scale_a t as three bfloat16 values, [M][3][Rp]
    __nv_bfloat16* terms;
    int mask_blocks, K, ldm;
    DropKey key;
    uint32_t* mask;             // [M][ldm]
};

// perm: rows sorted by adapter; start[a]: where adapter a's begin, start[adapters]: how many there are.  A block per adapter.
__device__ __forceinline__ void prep_sort(const AdRows& r, int* __restrict__ perm, int* __restrict__ start, int a) {
    __shared__ long long sum_own[8];
    __shared__ int sum_less[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
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
    if (lane == 0) { sum_less[warp] = (int)min(less, (long long)r.M); sum_own[warp] = own; }
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
        long long incl = n;                                      // of offsets that decrease every request may have all M rows: 32 bits would not hold the sum
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        __syncthreads();
        if (lane == 31) sum_own[warp] = incl;
        __syncthreads();
        long long at = incl - n, total = 0;
        for (int w = 0; w < 8; ++w) { if (w < warp) at += sum_own[w]; total += sum_own[w]; }
        // a warp writes the rows of its own segments one after the other
        for (unsigned some = __ballot_sync(0xffffffffu, n > 0); some; some &= some - 1) {
            const int k = __ffs(some) - 1;
            const int f = __shfl_sync(0xffffffffu, first, k);
            const long long to = base + __shfl_sync(0xffffffffu, at, k);
            const long long len = min((long long)__shfl_sync(0xffffffffu, n, k), r.M - to);        // 0 or less behind the end of the list
            for (int i = lane; i < len; i += 32) perm[to + i] = f + i;
        }
        base += total;
    }
}

// A 32 x 32 tile of an adapter's second factor, turned, with zeros behind its rows.
__device__ __forceinline__ void prep_turn(const PrepParams& p, int block) {
    __shared__ __nv_bfloat16 tile[32][33];
    const int bx = block % p.turn_x, by = block / p.turn_x % p.turn_y, a = block / (p.turn_x * p.turn_y);
    const int n0 = bx * 32, r0 = by * 32, tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    for (int i = ty; i < 32; i += 8) {
        const int n = n0 + i, r = r0 + tx;
        tile[i][tx] = n < p.N && r < p.R ? p.b[((size_t)a * p.N + n) * p.R + r] : __float2bfloat16_rn(0.f);
    }
    __syncthreads();
    for (int i = ty; i < 32; i += 8) {
        const int r = r0 + i, n = n0 + tx;
        if (r < p.R && n < (int)p.ldb) p.bt[((size_t)a * p.R + r) * p.ldb + n] = tile[tx][i];
    }
}
// 32 rows of scale_a t as sums of three bfloat16 values.
__device__ __forceinline__ void prep_terms(const PrepParams& p, int block) {
    __shared__ float scales[32];
    __shared__ int ids[32];
    const int m0 = block * 32;
    if (threadIdx.x < 32) {
        const int id = adapter_of_warp_row(p.rows, m0, (int)threadIdx.x);
        ids[threadIdx.x] = id;
        scales[threadIdx.x] = id >= 0 && p.scale ? __ldg(p.scale + id) : 1.f;
    }
    __syncthreads();
    const int pairs = p.Rp >> 1;
    for (int i = threadIdx.x; i < 32 * pairs; i += 256) {
        const int row = i / pairs, r = 2 * (i - row * pairs);
        if (ids[row] < 0) continue;
        const float* src = p.t + (size_t)(m0 + row) * p.R + r;
        uint32_t* dst = reinterpret_cast<uint32_t*>(p.terms + (size_t)(m0 + row) * 3 * p.Rp + r);
        uint32_t u[3];
        split3(r < p.R ? src[0] * scales[row] : 0.f, r + 1 < p.R ? src[1] * scales[row] : 0.f, u[0], u[1], u[2]);
#pragma unroll
        for (int k = 0; k < 3; ++k) dst[(size_t)k * pairs] = u[k];
    }
}
// What the dropout keeps, 64 channels of a row to a thread: the generator's rounds depend on one another, eight draws do not.
__device__ __forceinline__ void prep_mask(const PrepParams& p, int block) {
    const unsigned long long off = drop_offset(p.key);
    const int per = p.ldm >> 1;
    const size_t n = (size_t)p.rows.M * per, stride = (size_t)p.mask_blocks * 256;
    for (size_t i = (size_t)block * 256 + threadIdx.x; i < n; i += stride) {
        const size_t row = i / per;
        const unsigned long long e = (unsigned long long)row * p.K + 64 * (i - row * per);
        const int sh = (int)(e & 7);
        unsigned long long v = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) v |= (unsigned long long)drop_bits8(p.key, off, (e >> 3) + k) << (8 * k);
        if (sh) v = v >> sh | (unsigned long long)drop_bits8(p.key, off, (e >> 3) + 8) << (64 - sh);
        reinterpret_cast<unsigned long long*>(p.mask)[i] = v;
    }
}
__global__ void __launch_bounds__(256) adapter_prep_kernel(const PrepParams p) {
    const int b = blockIdx.x;
    grid_launch_dependents();
    if (b < p.sort_blocks) prep_sort(p.rows, p.perm, p.start, b);
    else if (b < p.sort_blocks + p.turn_blocks) prep_turn(p, b - p.sort_blocks);
    else if (b < p.sort_blocks + p.turn_blocks + p.term_blocks) prep_terms(p, b - p.sort_blocks - p.turn_blocks);
    else prep_mask(p, b - p.sort_blocks - p.turn_blocks - p.term_blocks);
}
int adapter_prep_run(const AdRows& rows, int* perm, int* start, int N, int R, int Rp, const __nv_bfloat16* b, __nv_bfloat16* bt, size_t ldb, const float* t,
                     const float* scale, __nv_bfloat16* terms, const DropKey& key, int K, uint32_t* mask, int ldm, cudaStream_t s) {
    PrepParams p = {};
    p.key = key; p.K = K; p.ldm = ldm; p.mask = mask;
    p.mask_blocks = mask ? (int)std::min<size_t>(((size_t)rows.M * (ldm >> 1) + 255) / 256, (size_t)num_sms() * 32) : 0;
    p.rows = rows;
    p.perm = perm; p.start = start; p.N = N; p.R = R; p.Rp = Rp; p.b = b; p.bt = bt; p.ldb = ldb; p.t = t; p.scale = scale; p.terms = terms;
    p.sort_blocks = perm ? rows.adapters : 0;
    p.turn_x = (int)((ldb + 31) / 32);
    p.turn_y = (R + 31) / 32;
    const long long turn = bt ? (long long)p.turn_x * p.turn_y * rows.adapters : 0, term = terms ? (rows.M + 31) / 32 : 0;
    const long long blocks = p.sort_blocks + turn + term + p.mask_blocks;
    if (blocks > 0x7fffffffll) return DR_ERR_UNSUPPORTED;
    p.turn_blocks = (int)turn; p.term_blocks = (int)term;
    adapter_prep_kernel<<<(unsigned)blocks, 256, 0, s>>>(p);
    count_launch();
    return launch_status();
}

// ---- the products ---------------------------------------------------------------------------------------------------------------------
constexpr int GR_THREADS = 384, GR_MASKERS = 128;      // warps 0, 2, 3 load, 1 issues MMAs, 4-11 drain; 12-15 mask, where there is a dropout
constexpr int GR_ROWS = 64;                            // rows of a stage
constexpr int GR_MAX_STAGES = 8;
constexpr int GR_SMEM = 222 * 1024;
constexpr int GR_BOX = GR_ROWS * 128;
// Rows summed in TMEM at a time: the tensor cores cut their sums off instead of rounding them, so an error grows with the number of MMAs in a row;
// longer sums are added up in float32 by the drain.  Sums of 16384 rows and more are off by 5e-7 so, da
// (whose u is such a sum too) by 9e-7; with all 2048 rows of an adapter in one it was over 1e-6.
constexpr int GR_CHAIN = 512;

struct GradParams {
    int M, R, Rp, adapters, splits;
    int tiles;                  // accumulators of 128 columns
    int rn, N, acc_cols, tmem_cols;     // r of a chunk of ranks (a multiple of 8), accumulator columns (three terms of them), their place in TMEM
    int rchunks, p_boxes, stages, stage_bytes;
    const int *perm, *start;
    int blocks0;                // column blocks of the first job
    int* status;
    struct Job {
        int C, swap, vec;           // vec: swapped rows of whole 16 bytes
        const uint32_t* mask;       // rows of ldm words
        int ldm;
        float *part, *out;
    } job[2];
};
struct GradShared {
    uint64_t landed[GR_MAX_STAGES], full[GR_MAX_STAGES], empty[GR_MAX_STAGES], tfull, tempty;
    uint32_t tmem;
    int abort;
};

// four rows of 64 columns from x on
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, int r0, int r1, int r2, int r3) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(dst),
                 "l"(map), "r"(bar), "r"(x), "r"(r0), "r"(r1), "r"(r2), "r"(r3)
                 : "memory");
}
__device__ __forceinline__ uint32_t sdesc_mn(uint32_t smem_addr) { return ((smem_addr & 0x3FFFFu) >> 4) | ((uint32_t)(GR_BOX >> 4) << 16); }

struct GradMaps { CUtensorMap z[2][3], p[2][3]; };              // of both jobs: for gathers, boxes of 16 and of 64 rows

// rows of a share: whole groups of 16 where there are many
__device__ __forceinline__ int grad_share(int total, int splits) {
    const int n = (total + splits - 1) / splits;
    return n >= 64 ? (n + 15) & ~15 : n;
}
// Shares and adapters of a CTA, in order: calls f(adapter, first sorted row, row behind the last, whole adapter?)
template <class F>
__device__ __forceinline__ void grad_ranges(const GradParams& p, int split, F f) {
    const int total = min(max(__ldg(p.start + p.adapters), 0), p.M);
    const int share = grad_share(total, p.splits);
    const int from = min(split * share, total), to = min(from + share, total);
    if (from >= to) return;
    int lo = 0, hi = p.adapters;                       // the first adapter whose rows reach beyond `from`
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(p.start + mid + 1) <= from) lo = mid + 1;
        else hi = mid;
    }
    for (int a = lo; a < p.adapters; ++a) {
        const int u0 = __ldg(p.start + a), v0 = min(__ldg(p.start + a + 1), total);
        if (u0 >= to) break;
        if (u0 < v0 && !f(a, max(from, u0), min(to, v0), u0 >= from && v0 <= to)) return;
    }
}

template <bool DROP>
__global__ void __launch_bounds__(GR_THREADS + (DROP ? GR_MASKERS : 0), 1)
adapter_grad_kernel(const __grid_constant__ GradMaps maps, const __grid_constant__ GradParams p) {
    extern __shared__ uint8_t gr_raw[];
    __shared__ GradShared sh;
    const uint32_t ring = (smem_u32(gr_raw) + 1023u) & ~1023u;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int which = (int)blockIdx.x >= p.blocks0;
    const GradParams::Job& j = p.job[which];
    const bool drop = DROP && j.mask;
    const int split = blockIdx.y, r0 = (int)blockIdx.z * p.rn, rn = min(p.rn, p.Rp - r0);
    const int c0 = ((int)blockIdx.x - (which ? p.blocks0 : 0)) * p.tiles * 128;
    volatile int* abort_flag = &sh.abort;
    if (threadIdx.x == 0) {
        for (int i = 0; i < p.stages; ++i) { mbar_init(&sh.landed[i], 1); mbar_init(&sh.full[i], GR_MASKERS / 32); mbar_init(&sh.empty[i], 1); }
        mbar_init(&sh.tfull, 1);
        mbar_init(&sh.tempty, 8);
        sh.abort = 0;
        fence_barrier_init();
        for (int k = 0; k < 3; ++k) { prefetch_tensormap(&maps.z[which][k]); prefetch_tensormap(&maps.p[which][k]); }
    }
    if (warp == 1) { tmem_alloc(&sh.tmem, (uint32_t)p.tmem_cols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_launch_dependents();
    grid_dependency_wait();                            // the lists, u and t's terms are the work of the kernels in front
    const uint32_t tmem = sh.tmem;
    const uint32_t landed0 = smem_u32(&sh.landed[0]), full0 = smem_u32(drop ? &sh.full[0] : &sh.landed[0]), empty0 = smem_u32(&sh.empty[0]);
    auto give_up = [&](int site) {
        if (!*abort_flag) report_timeout(p.status, site, split);
        *abort_flag = 1;
    };
    auto rows_of = [&](int i, int v, int (&rows)[2]) {         // two of the 64 rows from sorted row i on to a lane; M: none
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int at = i + 32 * h + lane;
            rows[h] = at < v ? (int)min((unsigned)__ldg(p.perm + at), (unsigned)(p.M - 1)) : p.M;
        }
    };

    if (warp < 4 && warp != 1) {
        // ---------------------------------------------------------------- loads: a lane has four rows, eight lanes sixteen; each warp every third box
        const int w = warp ? warp - 1 : 0;
        const int group = lane & 15, boxes = 2 * p.tiles + p.p_boxes;
        int s = 0;
        uint32_t ph = 0;
        grad_ranges(p, split, [&](int, int u, int v, bool) {
            int rows[2], next[2];
            rows_of(u, v, rows);
            for (int i = u; i < v; i += GR_ROWS) {
                rows_of(i + GR_ROWS, v, next);                 // on their way during this tile
                int r[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int from = 4 * (group & 7) + k;
                    const int a = __shfl_sync(0xffffffffu, rows[0], from), b = __shfl_sync(0xffffffffu, rows[1], from);
                    r[k] = group < 8 ? a : b;
                }
                if (!__all_sync(0xffffffffu, mbar_wait_u32(empty0 + 8 * s, ph ^ 1, abort_flag))) { give_up(101); return false; }
                if (lane == 0 && w == 0) mbar_expect_tx_u32(landed0 + 8 * s, (uint32_t)p.stage_bytes);
                __syncwarp();
                const int lead = __shfl_sync(0xffffffffu, r[0], lane & ~3);
                const bool run = r[0] == lead + 4 * (lane & 3) && r[1] == r[0] + 1 && r[2] == r[0] + 2 && r[3] == r[0] + 3 && r[3] < p.M;
                const unsigned runs = __ballot_sync(0xffffffffu, run);
                const bool sixteen = (runs >> (lane & ~3) & 0xFu) == 0xFu;
                const int zero = __shfl_sync(0xffffffffu, r[0], 0);
                const bool all = runs == 0xffffffffu && __all_sync(0xffffffffu, lead == zero + 16 * (group >> 2));
                auto from_x = [&](int b) { const int pb = b - 2 * p.tiles; return pb < 0 ? c0 + 64 * b : p.rchunks > 1 ? pb * p.Rp + r0 : 64 * pb; };
                const uint32_t tile = ring + (uint32_t)s * p.stage_bytes, bar = landed0 + 8 * s;
                if (all) {
                    if (lane == 0)
                        for (int b = w; b < boxes; b += 3)
                            tma_load_2d_u32<false>(tile + (uint32_t)b * GR_BOX, b < 2 * p.tiles ? &maps.z[which][2] : &maps.p[which][2], bar, from_x(b), zero, 1u);
                } else {
                    // neighbours: the eight lanes of the sixteen rows take every eighth of the warp's boxes; others: each lane its own rows of every second
                    const uint32_t dst = tile + (sixteen ? 2048u * (group >> 2) : 512u * group);
                    const int first = sixteen ? (lane >> 4) * 4 + (lane & 3) : lane >> 4, step = sixteen ? 8 : 2;
                    for (int b = w + 3 * first; b < boxes; b += 3 * step) {
                        const int k = b < 2 * p.tiles;
                        if (sixteen) tma_load_2d_u32<false>(dst + (uint32_t)b * GR_BOX, k ? &maps.z[which][1] : &maps.p[which][1], bar, from_x(b), lead, 1u);
                        else tma_gather4(dst + (uint32_t)b * GR_BOX, k ? &maps.z[which][0] : &maps.p[which][0], bar, from_x(b), r[0], r[1], r[2], r[3]);
                    }
                }
                __syncwarp();
                if (++s == p.stages) { s = 0; ph ^= 1; }
                rows[0] = next[0]; rows[1] = next[1];
            }
            return true;
        });
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMAs
        if (lane == 0) {
            const uint32_t idesc = make_idesc_bf16(128, p.N) | (1u << 15) | (1u << 16);          // both with the contraction index as rows
            int s = 0, n = 0;
            uint32_t ph = 0;
            grad_ranges(p, split, [&](int, int u, int v, bool) {
                for (int chain = u; chain < v; chain += GR_CHAIN, ++n) {
                    if (!mbar_wait(&sh.tempty, (uint32_t)(n & 1) ^ 1, abort_flag)) { give_up(102); return false; }
                    tc_fence_after();
                    uint32_t accum = 0;
                    const int end = min(v, chain + GR_CHAIN);
                    for (int i = chain; i < end; i += GR_ROWS) {
                        if (!mbar_wait_u32(full0 + 8 * s, ph, abort_flag)) { give_up(103); return false; }
                        tc_fence_after();
                        const uint32_t z = ring + (uint32_t)s * p.stage_bytes, b = sdesc_mn(z + (uint32_t)(2 * p.tiles) * GR_BOX);
                        const int n16 = (min(end - i, GR_ROWS) + 15) >> 4;
                        for (int t = 0; t < p.tiles; ++t) {
                            const uint32_t a = sdesc_mn(z + (uint32_t)(2 * t) * GR_BOX);
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                umma_bf16_lo<false>(tmem + (uint32_t)(t * p.acc_cols), a + 128 * k, b + 128 * k, idesc, accum | (uint32_t)(k > 0), k < n16 ? 1u : 0u);
                        }
                        accum = 1;
                        umma_commit_u32<false>(empty0 + 8 * s);
                        if (++s == p.stages) { s = 0; ph ^= 1; }
                    }
                    umma_commit(&sh.tfull);
                }
                return true;
            });
        }
        __syncwarp();
    } else if (DROP && warp >= 12) {
        // ---------------------------------------------------------------- mask: clears the dropped values of a tile
        if (drop) {
            // A thread has one row's 64 columns of a box, of every second box; the next tile's bits are on their way during this one.
            const int r = ((int)threadIdx.x - GR_THREADS) & 63, box0 = ((int)threadIdx.x - GR_THREADS) >> 6, boxes = min(2 * p.tiles, (j.C - c0 + 63) >> 6);
            int s = 0;
            uint32_t ph = 0;
            auto row_of = [&](int i, int v) { return i + r < v ? (int)min((unsigned)__ldg(p.perm + i + r), (unsigned)(p.M - 1)) : -1; };
            auto bits_of = [&](int row, uint2 (&bits)[4]) {
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int b = box0 + 2 * k;
                    bits[k] = make_uint2(0, 0);
                    if (row >= 0 && b < boxes) bits[k] = __ldcg(reinterpret_cast<const uint2*>(j.mask + (size_t)row * j.ldm + (c0 >> 5)) + b);
                }
            };
            grad_ranges(p, split, [&](int, int u, int v, bool) {
                uint2 bits[4], next[4];
                bits_of(row_of(u, v), bits);
                int row = row_of(u + GR_ROWS, v);
                for (int i = u; i < v; i += GR_ROWS) {
                    bits_of(row, next);
                    row = row_of(i + 2 * GR_ROWS, v);
                    if (!__all_sync(0xffffffffu, mbar_wait_u32(landed0 + 8 * s, ph, abort_flag))) { give_up(105); return false; }
                    uint8_t* const tile = gr_raw + (ring + (uint32_t)s * p.stage_bytes - smem_u32(gr_raw)) + r * 128;
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        if (box0 + 2 * k >= boxes) break;
                        uint4* const at = reinterpret_cast<uint4*>(tile + (box0 + 2 * k) * GR_BOX);
                        uint4 x[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) x[q] = at[q ^ (r & 7)];
#pragma unroll
                        for (int q = 0; q < 8; ++q) at[q ^ (r & 7)] = drop_apply8(x[q], (q < 4 ? bits[k].x : bits[k].y) >> (8 * (q & 3)) & 0xFFu);
                    }
                    #pragma unroll
                    for (int k = 0; k < 4; ++k) bits[k] = next[k];
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.full[s]);
                    if (++s == p.stages) { s = 0; ph ^= 1; }
                }
                return true;
            });
        }
    } else if (warp >= 4) {
        // ---------------------------------------------------------------- drain: lane = column of z, accumulator column = term and r
        // Two warps to a quarter of the lanes: a tile each, or every other eight r of the only tile.  Sums over chains stay in registers.
        constexpr int BLOCKS = 10;                              // of eight r: two tiles of 40 (four tiles of at most 128 columns), one of 64
        const int q = warp & 3, side = (warp - 4) >> 2;
        const int r8 = rn >> 3, mine = p.tiles > 1 ? (p.tiles >> 1) * r8 : (r8 + 1 - side) >> 1;
        int n = 0;
        auto tile_of = [&](int b) { return p.tiles > 1 ? side + 2 * (b >= r8 ? 1 : 0) : 0; };
        auto r_of = [&](int b) { return p.tiles > 1 ? 8 * (b >= r8 ? b - r8 : b) : 8 * (2 * b + side); };
        // eight r of a column: to [R][C] or, where swapped, [C][R]
        auto put = [&](float* to, int c, int r, const float* x) {
            float* at = to + (j.swap ? (size_t)c * p.R + r : (size_t)r * j.C + c);
            if (j.vec) {
                reinterpret_cast<float4*>(at)[0] = make_float4(x[0], x[1], x[2], x[3]);
                if (r + 4 < p.R) reinterpret_cast<float4*>(at)[1] = make_float4(x[4], x[5], x[6], x[7]);
                return;
            }
            const size_t step = j.swap ? 1 : j.C;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (r + i < p.R) at[i * step] = x[i];
        };
        grad_ranges(p, split, [&](int a, int u, int v, bool whole) {
            float acc[BLOCKS][8];
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[b][i] = 0.f;
            for (int chain = u; chain < v; chain += GR_CHAIN, ++n) {
                if (!__all_sync(0xffffffffu, mbar_wait(&sh.tfull, (uint32_t)(n & 1), abort_flag))) { give_up(104); return false; }
                tc_fence_after();
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    if (b >= mine) break;
                    const uint32_t at = tmem + (uint32_t)(tile_of(b) * p.acc_cols + r_of(b)) + ((uint32_t)(q * 32) << 16);
                    uint32_t x[8], y[8], z[8];
                    tmem_ld_x8(at + 2 * p.rn, x);
                    tmem_ld_x8(at + p.rn, y);
                    tmem_ld_x8(at, z);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[b][i] += (__uint_as_float(x[i]) + __uint_as_float(y[i])) + __uint_as_float(z[i]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.tempty);
            }
            float* to = whole ? j.out + (size_t)a * p.R * j.C : j.part + (size_t)(split + a) * p.R * j.C;
#pragma unroll
            for (int b = 0; b < BLOCKS; ++b) {
                const int c = c0 + 128 * tile_of(b) + 32 * q + lane;
                if (b < mine && c < j.C) put(to, c, r0 + r_of(b), acc[b]);
            }
            return true;
        });
        // adapters without rows, shared out over the splits
        const float zero[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        for (int a = split; a < p.adapters; a += p.splits) {
            if (__ldg(p.start + a) < __ldg(p.start + a + 1)) continue;
            for (int b = 0; b < mine; ++b) {
                const int c = c0 + 128 * tile_of(b) + 32 * q + lane;
                if (c < j.C) put(j.out + (size_t)a * p.R * j.C, c, r0 + r_of(b), zero);
            }
        }
    }
    tc_fence_before();
    ap_settle(abort_flag);
    if (warp == 1) tmem_dealloc(tmem, (uint32_t)p.tmem_cols);
}

// Adapters whose rows lie in more than one share: their partial sums in order.
__global__ void __launch_bounds__(256) adapter_grad_join_kernel(const __grid_constant__ GradParams p) {
    const GradParams::Job& j = p.job[blockIdx.z];
    grid_dependency_wait();
    if (!j.out) return;
    const int a = blockIdx.y;
    const int total = min(max(__ldg(p.start + p.adapters), 0), p.M);
    const int share = grad_share(total, p.splits);
    const int u = __ldg(p.start + a), v = min(__ldg(p.start + a + 1), total);
    if (u >= v) return;
    const int s0 = u / share, s1 = (v - 1) / share;
    if (s0 == s1) return;
    const size_t n = (size_t)p.R * j.C, stride = (size_t)gridDim.x * 256;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += stride) {
        float s = 0.f;
        const float* part = j.part + (size_t)(s0 + a) * n + i;
#pragma unroll 4
        for (int k = s0; k <= s1; ++k, part += n) s += *part;
        j.out[(size_t)a * n + i] = s;
    }
}

GradPlan adapter_grad_plan(int M, int R, int adapters, const int C[2]) {
    GradPlan g = {};
    const int Rp = (R + 7) / 8 * 8, sms = num_sms();
    g.rchunks = (Rp + 63) / 64;
    g.rn = g.rchunks == 1 ? Rp : 64;
    const int cols = (3 * g.rn + 31) / 32 * 32;               // of an accumulator
    // Columns of a CTA: as many as tensor memory has room for, fewer where that leaves SMs without rows.  Shares of at least 256 rows, or an adapter each: a
    // CTA takes 1.5 us for every adapter it meets
    const int most = std::max(std::max(1, (M + 255) / 256), std::min(adapters, M));
    for (g.tiles = 4; g.tiles > 1; g.tiles /= 2) {
        const int blocks = ((C[0] + 128 * g.tiles - 1) / (128 * g.tiles) + (C[1] + 128 * g.tiles - 1) / (128 * g.tiles)) * g.rchunks;
        if (g.tiles * cols <= 512 && (long long)blocks * most >= sms) break;
    }
    const int blocks = ((C[0] + 128 * g.tiles - 1) / (128 * g.tiles) + (C[1] + 128 * g.tiles - 1) / (128 * g.tiles)) * g.rchunks;
    g.splits = std::max(1, std::min(most, sms / blocks));
    size_t at = 0;
    auto take = [&](size_t& where, size_t bytes) { where = at; at += (bytes + 255) / 256 * 256; };
    take(g.perm, (size_t)M * 4);
    take(g.start, (size_t)(adapters + 1) * 4);
    take(g.terms, (size_t)M * 3 * Rp * 2);
    for (int k = 0; k < 2; ++k) take(g.part[k], g.splits > 1 ? (size_t)(g.splits + adapters - 1) * R * C[k] * 4 : 0);
    g.bytes = at;
    return g;
}

// rows of `cols` elements, `ld` apart, 64 columns and box_rows rows at a time
static int gr_map(CUtensorMap* map, const void* ptr, size_t rows, size_t cols, size_t ld, int box_rows) {
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {ld * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    return tmap_tiled(map, 2, ptr, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

int adapter_grad_run(const GradPlan& plan, const AdRows& rows, int R, const GradJob jobs[2], char* ws, bool overlap, cudaStream_t s) {
    GradParams p = {};
    p.M = rows.M; p.R = R; p.Rp = (R + 7) / 8 * 8; p.adapters = rows.adapters; p.splits = plan.splits;
    p.tiles = plan.tiles; p.rn = plan.rn; p.rchunks = plan.rchunks;
    p.N = (3 * plan.rn + 15) / 16 * 16;
    p.acc_cols = (p.N + 31) / 32 * 32;
    p.tmem_cols = 32;
    while (p.tmem_cols < p.acc_cols * p.tiles) p.tmem_cols *= 2;
    p.p_boxes = (3 * plan.rn + 63) / 64;
    p.stage_bytes = (2 * p.tiles + p.p_boxes) * GR_BOX;
    p.stages = std::min(GR_MAX_STAGES, GR_SMEM / p.stage_bytes);
    p.perm = (int*)(ws + plan.perm); p.start = (int*)(ws + plan.start);
    p.status = dev_status_ptr();
    int blocks[2];
    long long most = 0;
    for (int k = 0; k < 2; ++k) {
        const GradJob& g = jobs[k];
        p.job[k] = {g.C, g.swap, g.swap && (R & 3) == 0 && aligned16(g.out), g.mask, g.ldm, (float*)(ws + plan.part[k]), g.out};
        blocks[k] = g.out ? (g.C + 128 * p.tiles - 1) / (128 * p.tiles) : 0;
        if (g.out) most = std::max<long long>(most, (long long)R * g.C);
    }
    p.blocks0 = blocks[0];
    alignas(64) GradMaps maps = {};
    int rc = DR_OK;
    for (int k = 0; k < 2; ++k) {
        const GradJob& g = jobs[k];
        if (!g.out) continue;
        const int box[3] = {1, 16, GR_ROWS};
        for (int i = 0; i < 3 && rc == DR_OK; ++i) {
            rc = gr_map(&maps.z[k][i], g.z, p.M, g.C, g.ldz, box[i]);
            if (rc == DR_OK) rc = gr_map(&maps.p[k][i], g.p, p.M, 3 * (size_t)p.Rp, 3 * (size_t)p.Rp, box[i]);
        }
    }
    if (rc != DR_OK) return rc;
    const bool drop = jobs[0].out && jobs[0].mask;
    static PerDeviceFlag ready[2];
    if (!ready[drop].get()) {
        const cudaError_t e = drop ? cudaFuncSetAttribute(adapter_grad_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, GR_SMEM + 1024)
                                   : cudaFuncSetAttribute(adapter_grad_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, GR_SMEM + 1024);
        if (e != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
        ready[drop].set();
    }
    const dim3 grid((unsigned)(blocks[0] + blocks[1]), (unsigned)plan.splits, (unsigned)plan.rchunks);
    const int smem = 1024 + p.stages * p.stage_bytes;
    rc = drop ? start_kernel(adapter_grad_kernel<true>, grid, GR_THREADS + GR_MASKERS, 1, overlap, smem, s, maps, p)
              : start_kernel(adapter_grad_kernel<false>, grid, GR_THREADS, 1, overlap, smem, s, maps, p);
    if (rc == DR_OK && plan.splits > 1) {
        rc = start_kernel(adapter_grad_join_kernel, dim3((unsigned)std::min((most + 255) / 256, 512ll), (unsigned)rows.adapters, 2), 256, 1, true, 0, s, p);
    }
    return rc;
}

}  // namespace dr
