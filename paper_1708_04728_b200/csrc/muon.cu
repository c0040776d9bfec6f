// Orthogonalising an update by Newton-Schulz products, and the optimiser step that uses it:
//   X_0 = U / (|U|_F + eps),   A = X X^T,   X <- a X + (b A + c A A) X   (`steps` times),   O = X
//   v <- momentum v + g;  U = g + momentum v (Nesterov) or v;  w <- w - lr (sqrt(max(1, rows / cols)) O + decay w)
// X has n = min(rows, cols) rows and m columns: a taller U is worked on as its transpose.
//
// Arithmetic.  The products run on the tensor cores with float16 operands (11 significant bits) and float32 sums.  What keeps the
// result close to the formula is what is NOT rounded to 11 bits:
//  - X is carried as a pair of float16, X = (hi + lo) / 4096 (22 bits); the products read hi, the term a X reads both.
//  - A is split into its diagonal and the rest, A = D + E, D in float32:
//      A A = E E + D E + E D + D D,  so only E, small where X is nearly orthogonal, is rounded (and only for E E);
//    likewise the polynomial b A + c A A = diag + F:  X <- (a + diag) X + F X with a row factor in float32.
//    With the whole of A in float16 the relative error of O is 2e-3 .. 4e-3 (random matrices); with the split 1e-4 .. 9e-4, at most
//    1.3e-3 (512 rows) .. 2.3e-3 (130 rows, two steps at a time) for spectra over up to six decades, 1.2e-3 (512) .. 3.8e-3 (65 rows) for
//    ranks of 2 .. 16, and 1e-3 (512) .. 8e-3 (65 rows) for a single direction, where rounding errors do not average.
//  - A and E E are symmetric.  Where a group has a CTA for every tile, all are computed; otherwise those that reach the lower triangle, and
//    mirrored.  (Products of two different polynomials, two steps at a time, are symmetric up to rounding in the first case.)
// bfloat16 operands would cost 2e-3 .. 6e-3 even so: more than the rounding of O to bfloat16 itself.
//
// Execution.  One persistent kernel runs all products of a matrix: a group of G CTAs (one per SM) works through the phases
// A -> F -> X of every step and meets at a barrier between them; a batch is spread over the groups.  Inside a phase a CTA is a
// pipeline: one warp loads 128-deep operand slices by TMA, two issue tcgen05.mma into one of two sets of accumulators in
// tensor memory, eight drain the other one.  A group of up to 16 CTAs is a thread-block cluster and uses its barrier, where the device holds
// a cluster for every matrix and a power of two of CTAs leaves at most a quarter of them unused; others are launched cooperatively and
// count arrivals in global memory.  Where A has few tiles, its long axis is divided: over the CTAs of a
// cluster that exchange their parts through each other's shared memory, or over all CTAs with a phase more to sum the parts.
//
// Measured on a B200, five steps; flops executed, with A and A A by their lower triangles, against 1650 TFLOP/s of a bfloat16 product:
//   4096 x 9216   2.07 .. 2.48 ms (the clock falls with the power drawn), 0.63 .. 0.52 of that rate (2147 GFLOP, two steps of X at a time; the
//                 formula's 2663 would be 0.78 .. 0.65); the plain form in float32 takes 62.7 ms.  A pair's slice is 512 cycles of MMAs against
//                 700 of hand-over by its only issuing thread and as many for its operands out of L2; then whole rounds of tiles.
//   2048 x 2048   336 us, 0.31: 64 tiles of 256 x 256 for 74 pairs, drains of 8 us behind MMAs of 10.
//   1000 x 2048   176 us, 512 x 13200 with the optimiser's step 254 us, 512 x 2048 119 us, 6 x 256 x 2304 156 us (with the step 170), 192 x 576 101 us: 15 dependent
//                 phases of 6 to 20 us each.  A phase is a barrier 1.3 .. 1.9 us, 0.5 .. 1 to its first MMA's operands, 0.8 of TMA latency, the MMAs, and
//                 a drain of 1.3 .. 3; where all SMs load operands, the way out of L2 (12 TB/s).
#include <algorithm>
#include <cmath>
#include <cstring>

#include "muon_common.cuh"

namespace dr {

constexpr int NS_THREADS = 384;             // warp 0: TMA, warps 1 and 2: MMA, warps 4 - 11: drain, two for each quarter of the accumulator's rows
constexpr int NS_STAGES = 8;                // at most
constexpr int NS_SMEM = NS_SMEM_ALL - 1024; // operand ring
constexpr int NS_CHUNK = 128 * 128;          // 128 rows x 64 float16
// 64-column chunks a stage is deep in the contraction: 2, since the issuing threads take 400 cycles to hand a stage over; 1 where two
// CTAs share tiles of 256 x 256, whose MMAs take longer than that and want more stages of the same bytes (1.24 against 1.35 ms at 4096 x 4096)
__host__ __device__ constexpr int ns_depth(bool pair) { return pair ? 1 : 2; }
constexpr int NS_NORM_BLOCKS = 256;         // partial sums of squares at most

struct NsParams {
    NsInput in;
    int batch, steps;
    int n, m, ldx, lda;         // X: n x m, row stride ldx; A, E, F: n x n, row stride lda
    int G, groups, cluster, pair;
    int tr;                     // tile rows: 128, or 256 where two CTAs share a tile
    int nt_a, nt_s, nt_x;       // tile columns of the three products
    int tiles_a, tiles_s, tiles_x;
    int full_a, full_s;         // whether all tiles of A and of E E are computed, not those of the lower triangle alone
    int splits;                 // ranges of the long axis in A = X X^T whose parts meet in global memory, in a phase of its own
    int share;                  // or CTAs of a cluster that share a tile of it, a range each, and exchange parts through their shared memory
    int merge;                  // whether X takes two steps at a time
    int terms;                  // 1: hi hi;  3: hi hi + hi lo + lo hi
    int stages, stage_bytes;
    float coef[3 * DR_NS_MAX_STEPS];
    // per group
    __half *hi[2], *lo;
    // three n x n matrices: off-diagonal entries as float16 (and what that leaves out, with terms == 3), in float32, the diagonal
    __half *H[3], *L[2];
    float *W[3], *D[3], *part;
    double* norm;               // [groups][n_norm] where the kernel sums itself, [batch][n_norm] where ns_begin_kernel did
    int n_norm;
    unsigned* arrived;          // [groups]
    int* status;
};

enum { NS_A, NS_S, NS_X };
// Kernels: each CTA for itself, CTAs of a cluster that share A's tiles along the long axis, pairs of CTAs that share all tiles.  One kernel for the
// first two cost either 2 us in registers.
enum { NS_ALONE, NS_SHARE, NS_PAIR };
struct NsItem { int i, j, k0, k1, split, tile; };
struct NsShared {
    NsItem first[3];            // the CTA's first tile of each phase: found once, its divisions took 0.3 us of every phase
    uint64_t full[2 * NS_STAGES], empty[NS_STAGES], tfull[2], tempty[2];    // full: of each issuing warp
    uint32_t tmem_base;
    int abort;
    double red[NS_THREADS / 32];
};

// ------------------------------------------------------------------------------------------------ input and output
__global__ void __launch_bounds__(256) ns_begin_kernel(const NsInput in, double* norm, unsigned* arrived, int groups) {
    __shared__ double red[8];
    const size_t per = (size_t)in.rows * in.cols;
    if (blockIdx.y == 0 && blockIdx.x == 0)
        for (int i = threadIdx.x; i < groups; i += 256) arrived[i] = 0;
    const double s = ns_warp_sum(ns_momentum(in, blockIdx.y * per, per, (size_t)blockIdx.x * 256 + threadIdx.x, (size_t)gridDim.x * 256));
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        double t = 0.;
        for (int i = 0; i < 8; ++i) t += red[i];
        norm[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = t;
    }
}

// ------------------------------------------------------------------------------------------------ the products' tiles
// Tiles of tr rows x nt columns that reach the lower triangle, row by row.
__host__ __device__ __forceinline__ int ns_tri_row(int i, int n, int tr, int nt) { return min((n + nt - 1) / nt, (i * tr + tr - 1) / nt + 1); }
__device__ __forceinline__ void ns_tri_tile(int t, int n, int tr, int nt, int& i, int& j) {
    i = 0;
    for (int c; t >= (c = ns_tri_row(i, n, tr, nt)); ++i) t -= c;
    j = t;
}

template <int PHASE, bool PAIR>
__device__ __forceinline__ NsItem ns_item(const NsParams& p, int item) {
    NsItem it;
    it.split = 0;
    const int kb = ((PHASE == NS_A ? p.m : p.n) + 64 * ns_depth(PAIR) - 1) / (64 * ns_depth(PAIR));      // at most 1024; splits at most 148
    it.k0 = 0;
    it.k1 = kb;
    it.tile = item;
    if (PHASE == NS_A && p.share > 1) {
        it.tile = item / p.share;
        it.split = item - it.tile * p.share;
        it.k0 = kb * it.split / p.share;
        it.k1 = kb * (it.split + 1) / p.share;
    }
    if (PHASE == NS_A && p.splits > 1) {
        it.split = item / p.tiles_a;
        it.tile = item - it.split * p.tiles_a;
        it.k0 = kb * it.split / p.splits;
        it.k1 = kb * (it.split + 1) / p.splits;
    }
    if (PHASE == NS_X) {
        const int ni = (p.n + p.tr - 1) / p.tr;
        it.j = item / ni;
        it.i = item - it.j * ni;
    } else if (PHASE == NS_A ? p.full_a : p.full_s) {
        const int ni = (p.n + p.tr - 1) / p.tr;
        it.j = it.tile / ni;
        it.i = it.tile - it.j * ni;
    } else {
        ns_tri_tile(it.tile, p.n, p.tr, PHASE == NS_A ? p.nt_a : p.nt_s, it.i, it.j);
    }
    return it;
}

// the first `count` of CN float16 values of a row (a whole number of 16-byte pieces in all but the diagonal's tiles)
template <int CN>
__device__ __forceinline__ void ns_mirror(__half* p, int ld, int i, int c0, const uint32_t* h, int count) {
#pragma unroll
    for (int c = 0; c < CN; ++c)
        if (c < count) p[(size_t)(c0 + c) * ld + i] = __ushort_as_half((unsigned short)(h[c / 2] >> (16 * (c & 1))));
}
template <int CN>
__device__ __forceinline__ void ns_row_store(__half* p, const uint32_t* h, int count) {
    if (count == CN) {
#pragma unroll
        for (int c = 0; c < CN / 2; c += 4) *reinterpret_cast<uint4*>(p + 2 * c) = make_uint4(h[c], h[c + 1], h[c + 2], h[c + 3]);
    } else {
#pragma unroll
        for (int c = 0; c < CN; ++c)
            if (c < count) p[c] = __ushort_as_half((unsigned short)(h[c / 2] >> (16 * (c & 1))));
    }
}

// What the drain of A leaves for (row i, columns c0 .. c0 + CN - 1): A in float32, its diagonal, and the rest as float16.  `full`: every
// tile of the matrix is drained; otherwise those that reach the lower triangle, whose entries are mirrored.
template <int CN>
__device__ __forceinline__ void ns_emit_a(const NsParams& p, size_t mat, float* dvec, bool full, int i, int c0, float* v) {
    if (!full && c0 > i) return;
    float* A = p.W[0] + mat;
    const int last = full ? CN : min(CN, i - c0 + 1);
    if (last == CN) {
#pragma unroll
        for (int c = 0; c < CN; c += 8) st8f(A + (size_t)i * p.lda + c0 + c, v + c);
    } else {
#pragma unroll
        for (int c = 0; c < CN; ++c)
            if (c < last) A[(size_t)i * p.lda + c0 + c] = v[c];
    }
    if (c0 < (i | 31) + 1 && c0 + CN > (i & ~31)) {      // one of the warp's 32 rows meets its diagonal here: selects, and one store
        float d = 0.f;
#pragma unroll
        for (int c = 0; c < CN; ++c) {
            d = c0 + c == i ? v[c] : d;
            v[c] = c0 + c == i ? 0.f : v[c];
        }
        if (i >= c0 && i < c0 + CN) dvec[i] = d;
    }
    uint32_t h[CN / 2], l[CN / 2];
    ns_split<CN>(v, h, l);
    ns_row_store<CN>(p.H[0] + mat + (size_t)i * p.lda + c0, h, last);
    if (p.terms == 3) ns_row_store<CN>(p.L[0] + mat + (size_t)i * p.lda + c0, l, last);
    if (!full) {
        ns_mirror<CN>(p.H[0] + mat, p.lda, i, c0, h, last);
        if (p.terms == 3) ns_mirror<CN>(p.L[0] + mat, p.lda, i, c0, l, last);
        if (p.full_s) {
#pragma unroll
            for (int c = 0; c < CN; ++c)
                if (c0 + c < i) A[(size_t)(c0 + c) * p.lda + i] = v[c];
        }
    }
}

// A product of two of the n x n matrices, U V with U = diag(du) + Eu and V = diag(dv) + Ev: the tensor cores give Eu Ev (v), the rest is added
// here, du_i Ev_ij + Eu_ij dv_j and du_i dv_i.  `poly`: U = V = A, and the result is a + b A + c A A.  eu, ev: row i of U and V in
// float32, dj: V's diagonal at the columns.  `full` as above.
struct NsTriple { int u, v, to, poly, keep; };              // keep: the result is a factor of a later product, kept in float32 too
template <int CN>
__device__ __forceinline__ void ns_emit_n(const NsParams& p, const NsTriple& t, size_t mat, float* dvec, const float* coef, bool full, int i, int c0, float du, float dv, const float* dj,
                                          const float* eu, const float* ev, float* v) {
    if (!full && c0 > i) return;
    float diag = 0.f;
#pragma unroll
    for (int c = 0; c < CN; ++c) {
        diag = c0 + c == i ? v[c] : diag;
        float f = fmaf(du, ev[c], fmaf(eu[c], dj[c], v[c]));
        if (t.poly) f = fmaf(coef[1], eu[c], coef[2] * f);
        v[c] = c0 + c == i ? 0.f : f;
    }
    if (i >= c0 && i < c0 + CN) {
        diag = fmaf(du, dv, diag);
        dvec[i] = t.poly ? coef[0] + fmaf(coef[1], du, coef[2] * diag) : diag;
    }
    uint32_t h[CN / 2], l[CN / 2];
    ns_split<CN>(v, h, l);
    const int last = full ? CN : min(CN, i - c0 + 1);
    ns_row_store<CN>(p.H[t.to] + mat + (size_t)i * p.lda + c0, h, last);
    if (!full) ns_mirror<CN>(p.H[t.to] + mat, p.lda, i, c0, h, last);
    if (p.terms == 3) {
        ns_row_store<CN>(p.L[t.to] + mat + (size_t)i * p.lda + c0, l, last);
        if (!full) ns_mirror<CN>(p.L[t.to] + mat, p.lda, i, c0, l, last);
    }
    if (t.keep) {
        float* w = p.W[t.to] + mat + (size_t)i * p.lda + c0;
        if (last == CN) {
#pragma unroll
            for (int c = 0; c < CN; c += 8) st8f(w + c, v + c);
        } else {
#pragma unroll
            for (int c = 0; c < CN; ++c)
                if (c < last) w[c] = v[c];
        }
    }
}

// All operands are seen as [group][64-column chunk][row][64].  The first operand's boxes are 128 rows x a stage's depth in chunks.  The second's
// (b_*): 128 rows or, for the narrower tiles, 64; in the X product a stage's depth in rows x 2 chunks or 1.
struct NsMaps { CUtensorMap hi[2], lo, H[3], L[2], ba_hi[2], ba_lo, bs[3], bs_lo, bx_hi[2], bx_lo; };

template <int CN> __device__ __forceinline__ void tmem_ld(uint32_t addr, uint32_t* r) {
    if constexpr (CN == 8) tmem_ld_x8(addr, r);
    else tmem_ld_x16(addr, r);
}

// Where the roles of a CTA stand in their rings; kept from phase to phase.
struct NsPipe {
    int stage = 0;
    uint32_t phase = 0;
    int acc = 0;
    uint32_t acc_phase = 0;
    uint32_t mine = 0;          // an issuing warp: a bit for each stage, the parity of its own next fill
    __device__ __forceinline__ void next_stage(int stages) { if (++stage == stages) { stage = 0; phase ^= 1; } }
    __device__ __forceinline__ void next_acc() { if (++acc == 2) { acc = 0; acc_phase ^= 1; } }
};

template <int PHASE, int KIND>
__device__ __forceinline__ void ns_product(const NsParams& p, const NsMaps& maps, NsShared& sh, uint32_t smem, uint32_t tmem, NsPipe& pipe, int group, int rank, int src, const NsTriple triple, const float* coef) {
    constexpr bool PAIR = KIND == NS_PAIR, SHARE = KIND == NS_SHARE;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int nt = PHASE == NS_A ? p.nt_a : PHASE == NS_S ? p.nt_s : p.nt_x;
    const int items = PHASE == NS_A ? p.tiles_a * p.splits * p.share : PHASE == NS_S ? p.tiles_s : p.tiles_x;
    const int first = PAIR ? rank >> 1 : rank, step = PAIR ? p.G >> 1 : p.G, side = PAIR ? rank & 1 : 0;
    const uint32_t full0 = smem_u32(&sh.full[0]), empty0 = smem_u32(&sh.empty[0]), tfull0 = smem_u32(&sh.tfull[0]), tempty0 = smem_u32(&sh.tempty[0]);
    constexpr int D = ns_depth(PAIR);
    volatile int* abort_flag = &sh.abort;
    // The issuing threads: one elected lane of a warp whose number the compiler knows to be uniform, so that addresses and
    // descriptors stay in uniform registers.  With a plain lane test a hand-over of a stage cost 800 cycles, this way 400;
    // and a stage is two TMA boxes and up to eight MMAs for the same reason.
    if (warp == 0) {
        if (elect_one()) {
            const CUtensorMap *ah, *al, *bh, *bl;
            if (PHASE == NS_A) { ah = &maps.hi[src]; al = &maps.lo; bh = &maps.ba_hi[src]; bl = &maps.ba_lo; }
            else if (PHASE == NS_S) { ah = &maps.H[triple.u]; al = &maps.L[0]; bh = &maps.bs[triple.v]; bl = &maps.bs_lo; }
            else { ah = &maps.H[triple.u]; al = &maps.L[1]; bh = &maps.bx_hi[src]; bl = &maps.bx_lo; }
            const uint32_t bytes = PAIR ? (uint32_t)(2 * NS_CHUNK + nt * 128) : (uint32_t)(2 * NS_CHUNK + nt * 256);      // of a stage, pairs: of both CTAs
            bool ok = true;
            uint32_t ready = mbar_test_u32(empty0 + 8 * pipe.stage, pipe.phase ^ 1);
            for (int item = first; item < items && ok; item += step) {
                const NsItem it = item == first ? sh.first[PHASE] : ns_item<PHASE, PAIR>(p, item);
                const int ar = it.i * p.tr + side * 128, bc = it.j * nt + side * (nt / 2);
                uint32_t which = 0;                     // the warp that takes the slice
                for (int term = 0; term < p.terms && ok; ++term) {
                    const CUtensorMap* am = term == 2 ? al : ah;
                    const CUtensorMap* bm = term == 1 ? bl : bh;
                    for (int kb = it.k0; kb < it.k1; ++kb) {
                        if (!ready && !mbar_wait_slow_u32(empty0 + 8 * pipe.stage, pipe.phase ^ 1, abort_flag)) {
                            if (!*abort_flag) report_timeout(p.status, 71, item);
                            *abort_flag = 1;
                            ok = false;
                            break;
                        }
                        const uint32_t full = PAIR ? (full0 + 8 * pipe.stage) & PEER_BIT_MASK : full0 + which + 8 * pipe.stage;
                        if (!PAIR) which ^= 8 * NS_STAGES;
                        const uint32_t dst = smem + pipe.stage * p.stage_bytes;
                        if (side == 0) mbar_expect_tx_u32(full, bytes);
                        tma_load_4d_u32<PAIR>(dst, am, full, 0, ar, D * kb, group, 1u);
                        if (PHASE == NS_X) tma_load_4d_u32<PAIR>(dst + D * NS_CHUNK, bm, full, 0, D * 64 * kb, bc >> 6, group, 1u);
                        else tma_load_4d_u32<PAIR>(dst + D * NS_CHUNK, bm, full, 0, bc, D * kb, group, 1u);
                        pipe.next_stage(p.stages);
                        ready = mbar_test_u32(empty0 + 8 * pipe.stage, pipe.phase ^ 1);
                    }
                }
            }
        }
    } else if (warp <= 2) {
        // Two issuing warps (pairs of CTAs: one), each on every second slice into an accumulator of its own, which the drain adds: while one
        // hands a stage over, the other's MMAs run.  A warp sees only its own fills, and slices may land out of order, so each warp has a full
        // barrier of its own for every stage: on a common one, whose phases the other's fills complete too, the parity of a fill two phases ahead
        // is that of the one before it, and a wait for a slice could pass while the stage's last one was still on its way.
        const int which = warp - 1;
        if (side == 0 && (!PAIR || which == 0) && elect_one()) {
            // D float32, A and B float16; B of the X product lies with the contraction index as its rows
            const uint32_t idesc = (1u << 4) | ((uint32_t)(nt >> 3) << 17) | ((PAIR ? 16u : 8u) << 24) | (PHASE == NS_X ? 1u << 16 : 0u);
            const uint32_t b_chunk = (uint32_t)nt * 128u >> 4;      // 64 deep in K: a chunk of B's rows
            bool ok = true;
            for (int item = first; item < items && ok; item += step) {
                const NsItem it = item == first ? sh.first[PHASE] : ns_item<PHASE, PAIR>(p, item);
                if (!mbar_wait_u32(tempty0 + 8 * pipe.acc, pipe.acc_phase ^ 1, abort_flag)) {
                    if (!*abort_flag) report_timeout(p.status, 72, item);
                    *abort_flag = 1;
                    break;
                }
                tc_fence_after();
                const uint32_t acc = tmem + pipe.acc * 256 + (PAIR ? 0 : which * 128);
                uint32_t accumulate = 0;
                const int count = (it.k1 - it.k0) * p.terms;
                uint32_t ready = 0;
                for (int k = 0; k < count; ++k) {
                    if (!PAIR && (k & 1) != which) {
                        pipe.next_stage(p.stages);
                        continue;
                    }
                    if (!ready && !mbar_wait_u32(full0 + 8 * (pipe.stage + which * NS_STAGES), PAIR ? pipe.phase : (pipe.mine >> pipe.stage) & 1u, abort_flag)) {
                        if (!*abort_flag) report_timeout(p.status, 73, item);
                        *abort_flag = 1;
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t a = smem + pipe.stage * p.stage_bytes, b = a + D * NS_CHUNK, empty = empty0 + 8 * pipe.stage;
                    if (!PAIR) pipe.mine ^= 1u << pipe.stage;
                    pipe.next_stage(p.stages);
                    if (PAIR) ready = mbar_test_u32(full0 + 8 * pipe.stage, pipe.phase);    // asked before the MMAs, known after them
                    const uint32_t ad = sdesc_lo(a), bd = PHASE == NS_X ? (((b & 0x3FFFFu) >> 4) | ((D * 512u) << 16)) : sdesc_lo(b);
#pragma unroll
                    for (int ks = 0; ks < 4 * D; ++ks) {
                        umma_bf16_lo<PAIR>(acc, ad + (ks >> 2) * 1024 + (ks & 3) * 2, bd + (PHASE == NS_X ? ks * 128 : (ks >> 2) * b_chunk + (ks & 3) * 2), idesc, accumulate, 1u);
                        accumulate = 1;
                    }
                    umma_commit_u32<PAIR>(empty);
                }
                umma_commit_u32<PAIR>(tfull0 + 8 * pipe.acc);
                pipe.next_acc();
            }
        }
    } else if (warp >= 4) {
        const int q = warp & 3, part = (warp - 4) >> 2;
        const size_t mat = (size_t)group * p.n * p.lda, xm = (size_t)group * p.n * p.ldx;
        const size_t dg = (size_t)group * p.lda;
        for (int item = first; item < items; item += step) {
            const NsItem it = item == first ? sh.first[PHASE] : ns_item<PHASE, PAIR>(p, item);
            const int row = it.i * p.tr + side * 128 + q * 32 + lane;
            // Chunks of 16 columns (8 in the n x n products, which need more of each), alternating between the two warps of a quarter.  What a
            // chunk needs from memory is requested a chunk ahead, the first one's before the product is waited for.
            constexpr int CN = PHASE == NS_S ? 8 : 16;
            float factor = 0.f, dv = 0.f, dj_next = 0.f;    // NS_X: the row's factor; NS_S: the row's diagonal entries in U and V
            Half16 hn, ln;
            alignas(32) float un[8], vn[8];
            auto request = [&](int c) {
                const int col = it.j * nt + c;
                if (PHASE == NS_X && row < p.n && col < p.ldx) {
                    const size_t at = xm + (size_t)row * p.ldx + col;
                    hn = ld16h(p.hi[src] + at);
                    ln = ld16h(p.lo + at);
                }
                if (PHASE == NS_S && col < p.lda) {
                    dj_next = p.D[triple.v][dg + col + (lane & 7)];
                    if (row < p.n) {
                        ld8f(p.W[triple.u] + mat + (size_t)row * p.lda + col, un);
                        if (!triple.poly) ld8f(p.W[triple.v] + mat + (size_t)row * p.lda + col, vn);
                    }
                }
            };
            if (PHASE != NS_A && row < p.n) factor = p.D[triple.u][dg + row];
            if (PHASE == NS_S && row < p.n) dv = p.D[triple.v][dg + row];
            request(part * CN);
            const bool ok = __all_sync(0xffffffffu, mbar_wait_u32(tfull0 + 8 * pipe.acc, pipe.acc_phase, abort_flag));
            if (!ok) {
                if (!*abort_flag) report_timeout(p.status, 74, item);
                *abort_flag = 1;
                goto out;
            }
            tc_fence_after();
            const uint32_t acc = tmem + pipe.acc * 256 + ((uint32_t)(q * 32) << 16);
            const bool two = (it.k1 - it.k0) * p.terms > 1;         // both issuers had a stage
#pragma unroll 1
            for (int c = part * CN; c < nt; c += 2 * CN) {
                const int col = it.j * nt + c;
                uint32_t raw[CN], raw2[CN];
                alignas(32) float v[CN];
                __syncwarp();
                tmem_ld<CN>(acc + c, raw);
                if (!PAIR && two) tmem_ld<CN>(acc + 128 + c, raw2);
                float dj[8], eu[8], ev[8];
                Half16 h, l;
                if (PHASE == NS_X) { h = hn; l = ln; }
                if (PHASE == NS_S) {
#pragma unroll
                    for (int t = 0; t < 8; ++t) {
                        eu[t] = un[t];
                        ev[t] = triple.poly ? un[t] : vn[t];
                        dj[t] = __shfl_sync(0xffffffffu, dj_next, t);
                    }
                }
                if (PHASE != NS_A && c + 2 * CN < nt) request(c + 2 * CN);
                tmem_ld_wait();
#pragma unroll
                for (int t = 0; t < CN; ++t) v[t] = !PAIR && two ? __uint_as_float(raw[t]) + __uint_as_float(raw2[t]) : __uint_as_float(raw[t]);
                if (PHASE == NS_A && SHARE) {
                    const int cs = nt / p.share, owner = c / cs;
                    const uint32_t to = mapa_shared(smem + NS_SMEM - nt * 512, (p.cluster ? rank - it.split : 0) + owner) + (uint32_t)((it.split * cs + c - owner * cs) * 128 + q * 32 + lane) * 4;
#pragma unroll
                    for (int t = 0; t < CN; ++t) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + t * 512), "f"(v[t]) : "memory");
                } else if (PHASE == NS_A && !SHARE && p.splits > 1) {
                    float* out = p.part + (((size_t)group * p.splits + it.split) * p.tiles_a + it.tile) * nt * 128 + (size_t)c * 128 + q * 32 + lane;
#pragma unroll
                    for (int t = 0; t < CN; ++t) out[t * 128] = v[t];
                } else if (row < p.n) {
                    if constexpr (PHASE == NS_A) {
                        if (col < p.lda) {
#pragma unroll
                            for (int t = 0; t < CN; ++t) v[t] *= 1.f / (NS_SCALE * NS_SCALE);
                            ns_emit_a<CN>(p, mat, p.D[0] + dg, p.full_a, row, col, v);
                        }
                    } else if constexpr (PHASE == NS_S) {
                        if (col < p.lda) ns_emit_n<CN>(p, triple, mat, p.D[triple.to] + dg, coef, p.full_s, row, col, factor, dv, dj, eu, ev, v);
                    } else if (col < p.ldx) {
                        const size_t at = xm + (size_t)row * p.ldx + col;
#pragma unroll
                        for (int t = 0; t < 8; ++t) {
                            const float2 fh = half2_at(h.u[t]), fl = half2_at(l.u[t]);
                            v[2 * t] = fmaf(factor, fh.x + fl.x, v[2 * t]);
                            v[2 * t + 1] = fmaf(factor, fh.y + fl.y, v[2 * t + 1]);
                        }
                        ns_split<16>(v, h.u, l.u);
                        st16h(p.hi[src ^ 1] + at, h);
                        st16h(p.lo + at, l);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (PAIR) {
                if (lane == 0) mbar_arrive_leader(&sh.tempty[pipe.acc]);
            } else {
                if (lane == 0) mbar_arrive(&sh.tempty[pipe.acc]);
            }
            pipe.next_acc();
        }
    }
out:                                            // also after a wait that ran out: the whole warp goes on to the next barrier
    __syncwarp();
}

// All threads of the group's CTAs meet; what they wrote to global memory is visible to the others' loads, TMA included.
__device__ __forceinline__ void ns_group_sync(const NsParams& p, NsShared& sh, int group, unsigned& epoch) {
    asm volatile("fence.proxy.async;" ::: "memory");     // this thread's stores, before the other proxy's loads that follow the barrier
    if (p.G == 1) {
        __syncthreads();
    } else if (p.cluster) {
        cluster_sync_all();
    } else {
        __syncthreads();
        if (threadIdx.x == 0) {
            unsigned* c = p.arrived + group;
            asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(c) : "memory");
            const unsigned target = ++epoch * (unsigned)p.G;
            const long long t0 = clock64();
            for (;;) {
                unsigned seen;
                asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(c) : "memory");
                if (seen >= target || sh.abort) break;
                if (clock64() - t0 > WAIT_LIMIT_CYCLES) {
                    report_timeout(p.status, 75, (int)epoch);
                    sh.abort = 1;
                    break;
                }
            }
        }
        __syncthreads();
    }
}

// 8 (or 1) values of X_0 from U
template <int CN>
__device__ __forceinline__ void ns_put_x(__half* hi, __half* lo, NsFactor by, float* u) {
#pragma unroll
    for (int c = 0; c < CN; ++c) u[c] = u[c] * by.first * by.second;
    if (CN == 8) {
        uint32_t h[4], l[4];
        ns_split<8>(u, h, l);
        *reinterpret_cast<uint4*>(hi) = make_uint4(h[0], h[1], h[2], h[3]);
        *reinterpret_cast<uint4*>(lo) = make_uint4(l[0], l[1], l[2], l[3]);
    } else {
        *hi = __float2half_rn(u[0]);
        *lo = __float2half_rn(u[0] - __half2float(*hi));
    }
}
__device__ __forceinline__ void ns_get_x8(const __half* hi, const __half* lo, float* x) {
    const uint4 h = *reinterpret_cast<const uint4*>(hi), l = *reinterpret_cast<const uint4*>(lo);
    const uint32_t hu[4] = {h.x, h.y, h.z, h.w}, lu[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const float2 a = half2_at(hu[c]), b = half2_at(lu[c]);
        x[2 * c] = (a.x + b.x) * (1.f / NS_SCALE);
        x[2 * c + 1] = (a.y + b.y) * (1.f / NS_SCALE);
    }
}

// X_0 from U (LOAD) or the result from X.  Rows lie alike in both unless U is tall: a warp takes up to 1024 columns of a row.
// A tall U is transposed through a 64 x 64 tile in shared memory.
template <bool LOAD>
__device__ __forceinline__ void ns_convert(const NsParams& p, float* tile, int group, int rank, size_t base, int src, NsFactor by) {
    const NsInput& in = p.in;
    __half* hi = p.hi[src] + (size_t)group * p.n * p.ldx;
    __half* lo = p.lo + (size_t)group * p.n * p.ldx;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (!in.tall) {
        const int segs = (in.cols + 1023) / 1024, units = in.rows * segs;
        for (int u = rank * (NS_THREADS / 32) + warp; u < units; u += p.G * (NS_THREADS / 32)) {
            const int r = u / segs, c0 = (u - r * segs) * 1024, c1 = min(in.cols, c0 + 1024);
            const size_t x = (size_t)r * p.ldx, o = base + (size_t)r * in.cols;
            if (LOAD && c1 == in.cols)          // to a whole chunk of columns
                for (int c = c1 + lane; c < p.ldx; c += 32) hi[x + c] = lo[x + c] = __float2half_rn(0.f);
            if (in.vec) {
#pragma unroll 4
                for (int c = c0 + lane * 8; c < c1; c += 256) {
                    float f[8];
                    if (LOAD) {
                        ns_value<8>(in, o + c, f);
                        ns_put_x<8>(hi + x + c, lo + x + c, by, f);
                    } else {
                        ns_get_x8(hi + x + c, lo + x + c, f);
                        ns_put_o<8>(in, o + c, f);
                    }
                }
            } else {
#pragma unroll 4
                for (int c = c0 + lane; c < c1; c += 32) {
                    float f[1];
                    if (LOAD) {
                        ns_value<1>(in, o + c, f);
                        ns_put_x<1>(hi + x + c, lo + x + c, by, f);
                    } else {
                        f[0] = (__half2float(hi[x + c]) + __half2float(lo[x + c])) * (1.f / NS_SCALE);
                        ns_put_o<1>(in, o + c, f);
                    }
                }
            }
        }
        return;
    }
    const int tr = (in.rows + 63) / 64, tc = (in.cols + 63) / 64;
    for (int t = rank; t < tr * tc; t += p.G) {
        const int r0 = t / tc * 64, c0 = (t - t / tc * tc) * 64;
        // tile[row of U][column of U]
        auto user = [&]() {
            if (in.vec) {
                for (int e = threadIdx.x; e < 512; e += NS_THREADS) {
                    const int r = e >> 3, c = (e & 7) * 8;
                    if (r0 + r >= in.rows || c0 + c >= in.cols) continue;
                    const size_t o = base + (size_t)(r0 + r) * in.cols + c0 + c;
                    float f[8];
                    if (LOAD) ns_value<8>(in, o, f);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (LOAD) tile[r * 65 + c + k] = f[k];
                        else f[k] = tile[r * 65 + c + k];
                    }
                    if (!LOAD) ns_put_o<8>(in, o, f);
                }
            } else {
                for (int e = threadIdx.x; e < 4096; e += NS_THREADS) {
                    const int r = e >> 6, c = e & 63;
                    if (r0 + r >= in.rows || c0 + c >= in.cols) continue;
                    const size_t o = base + (size_t)(r0 + r) * in.cols + c0 + c;
                    float f[1];
                    if (LOAD) {
                        ns_value<1>(in, o, f);
                        tile[r * 65 + c] = f[0];
                    } else {
                        f[0] = tile[r * 65 + c];
                        ns_put_o<1>(in, o, f);
                    }
                }
            }
        };
        // X's rows are padded to 64 columns: whole vectors there
        auto inner = [&]() {
            for (int e = threadIdx.x; e < 512; e += NS_THREADS) {
                const int c = e & 63, r = (e >> 6) * 8;
                if (c0 + c >= in.cols) continue;
                const size_t x = (size_t)(c0 + c) * p.ldx + r0 + r;
                float f[8];
                if (!LOAD) ns_get_x8(hi + x, lo + x, f);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    if (LOAD) f[k] = r0 + r + k < in.rows ? tile[(r + k) * 65 + c] : 0.f;
                    else tile[(r + k) * 65 + c] = f[k];
                }
                if (LOAD) ns_put_x<8>(hi + x, lo + x, by, f);
            }
        };
        __syncthreads();
        if (LOAD) user();
        else inner();
        __syncthreads();
        if (LOAD) inner();
        else user();
    }
}

template <int KIND>
__global__ void __launch_bounds__(NS_THREADS, 1) ns_kernel(const __grid_constant__ NsMaps maps, const __grid_constant__ NsParams p) {
    constexpr bool PAIR = KIND == NS_PAIR, SHARE = KIND == NS_SHARE;
    extern __shared__ uint8_t ns_smem_raw[];
    __shared__ NsShared sh;
    const uint32_t smem = (smem_u32(ns_smem_raw) + 1023u) & ~1023u;
    float* tile = reinterpret_cast<float*>(ns_smem_raw + (smem - smem_u32(ns_smem_raw)));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = blockIdx.x / p.G, rank = blockIdx.x - group * p.G;
    if (cluster_lost(PAIR ? 2 : p.cluster ? p.G : SHARE ? p.share : 1, p.status)) return;
    if (threadIdx.x == 0) {
        for (int i = 0; i < NS_STAGES; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.full[NS_STAGES + i], 1); mbar_init(&sh.empty[i], 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.tfull[i], PAIR ? 1 : 2); mbar_init(&sh.tempty[i], PAIR ? 16 : 8); }
        sh.abort = 0;
        fence_barrier_init();
    }
    if (warp == 1) {
        if (PAIR) { tmem_alloc_pair(&sh.tmem_base, 512); tmem_relinquish_pair(); }
        else { tmem_alloc(&sh.tmem_base, 512); tmem_relinquish(); }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();               // both CTAs' barriers exist before any remote arrive
    tc_fence_after();
    const uint32_t tmem = sh.tmem_base;
    if (threadIdx.x == 0) {
        const int unit = PAIR ? rank >> 1 : rank;
        if (unit < p.tiles_a * p.splits * p.share) sh.first[NS_A] = ns_item<NS_A, PAIR>(p, unit);
        if (unit < p.tiles_s) sh.first[NS_S] = ns_item<NS_S, PAIR>(p, unit);
        if (unit < p.tiles_x) sh.first[NS_X] = ns_item<NS_X, PAIR>(p, unit);
    }
    NsPipe pipe;
    unsigned epoch = 0;
    // the columns that pad the n x n matrices to whole chunks take part in the products: zero (X's are zeroed where it is loaded)
    for (int i = rank * NS_THREADS + threadIdx.x; i < p.n * (p.lda - p.n); i += p.G * NS_THREADS) {
        const int r = i / (p.lda - p.n);
        const size_t at = ((size_t)group * p.n + r) * p.lda + p.n + (i - r * (p.lda - p.n));
        for (int k = 0; k < (p.merge ? 3 : 2); ++k) {
            p.H[k][at] = __float2half_rn(0.f);
            if (k == 0 || p.merge) p.W[k][at] = 0.f;
            if (p.terms == 3) p.L[k][at] = __float2half_rn(0.f);
            if (r == 0) p.D[k][(size_t)group * p.lda + p.n + i] = 0.f;
        }
    }
    const size_t per = (size_t)p.in.rows * p.in.cols;

    for (int b = group; b < p.batch; b += p.groups) {
        const size_t base = (size_t)b * per;
        const double* norm = p.norm + (size_t)b * p.n_norm;
        if (p.G == 1 || p.cluster) {            // no kernel in front has summed the squares: the group does
            double s = ns_warp_sum(ns_momentum(p.in, base, per, (size_t)rank * NS_THREADS + threadIdx.x, (size_t)p.G * NS_THREADS));
            if (lane == 0) sh.red[warp] = s;
            __syncthreads();
            if (threadIdx.x == 0) {
                s = 0.;
                for (int i = 0; i < NS_THREADS / 32; ++i) s += sh.red[i];
                p.norm[(size_t)group * p.n_norm + rank] = s;
            }
            norm = p.norm + (size_t)group * p.n_norm;
            ns_group_sync(p, sh, group, epoch);
        }
        double s = 0.;
        for (int i = lane; i < p.n_norm; i += 32) s += norm[i];
        ns_convert<true>(p, tile, group, rank, base, 0, ns_factor(ns_warp_sum(s), p.in.eps));
        ns_group_sync(p, sh, group, epoch);
        int src = 0;
        for (int k = 0; k < p.steps; src ^= 1) {
            const bool two = p.merge && k + 1 < p.steps;
            ns_product<NS_A, KIND>(p, maps, sh, smem, tmem, pipe, group, rank, src, NsTriple{}, nullptr);
            if (SHARE || (!PAIR && p.splits > 1)) {
                // The ranges' parts of A in order: a warp takes 32 rows x 8 columns, of those its CTA owns (share: their parts lie in its shared
                // memory) or of all.
                constexpr bool own = SHARE;
                if (own) cluster_sync_all();
                else ns_group_sync(p, sh, group, epoch);
                const int nt = p.nt_a, width = own ? nt / p.share : nt, parts = own ? p.share : p.splits;
                const int units = own ? (rank < p.tiles_a * p.share ? width / 2 : 0) : p.tiles_a * nt / 2;
                const size_t apart = own ? width * 128 : (size_t)p.tiles_a * nt * 128;
                for (int u = own ? warp : rank * (NS_THREADS / 32) + warp; u < units; u += own ? NS_THREADS / 32 : p.G * (NS_THREADS / 32)) {
                    const int t = u / (width / 2), rem = u - t * (width / 2), r = (rem & 3) * 32 + lane, c = (rem >> 2) * 8;
                    int i, j, col;
                    const float* in;
                    if (own) {
                        i = sh.first[NS_A].i;
                        j = sh.first[NS_A].j;
                        col = j * nt + sh.first[NS_A].split * width + c;
                        in = tile + (NS_SMEM - nt * 512) / 4;
                    } else {
                        ns_tri_tile(t, p.n, 128, nt, i, j);
                        col = j * nt + c;
                        in = p.part + ((size_t)group * p.splits * p.tiles_a + t) * nt * 128;
                    }
                    const int row = i * 128 + r;
                    in += (size_t)c * 128 + r;
                    alignas(32) float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                    for (int q = 0; q < parts; ++q, in += apart)
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += in[e * 128];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= 1.f / (NS_SCALE * NS_SCALE);
                    if (row < p.n && col < p.lda) ns_emit_a<8>(p, (size_t)group * p.n * p.lda, p.D[0] + (size_t)group * p.lda, p.full_a, row, col, v);
                }
            }
            ns_group_sync(p, sh, group, epoch);
            // A in 0.  One step: Q(A) in 1, X <- Q X.  Two: all factors are polynomials of A and commute, so the second step's A is Q A Q:
            // Q(A) in 1, Q A in 2, A' = (Q A) Q in 0, Q'(A') in 2, Q' Q in 0, X <- (Q' Q) X.
#pragma unroll 1
            for (int j = 0; j < (two ? 5 : 1); ++j) {
                const NsTriple t = j == 0 ? NsTriple{0, 0, 1, 1, two} : j == 1 ? NsTriple{1, 0, 2, 0, 1} : j == 2 ? NsTriple{2, 1, 0, 0, 1} : j == 3 ? NsTriple{0, 0, 2, 1, 1} : NsTriple{2, 1, 0, 0, 0};
                ns_product<NS_S, KIND>(p, maps, sh, smem, tmem, pipe, group, rank, src, t, p.coef + 3 * (k + (j == 3)));
                ns_group_sync(p, sh, group, epoch);
            }
            ns_product<NS_X, KIND>(p, maps, sh, smem, tmem, pipe, group, rank, src, NsTriple{two ? 0 : 1, 0, 0, 0, 0}, nullptr);
            ns_group_sync(p, sh, group, epoch);
            k += two ? 2 : 1;
        }
        ns_convert<false>(p, tile, group, rank, base, src, NsFactor{});
        ns_group_sync(p, sh, group, epoch);     // the buffers are free for the group's next matrix
    }
    if (sh.abort) {                             // copies and products in flight end within microseconds; then the CTA may go
        const long long t0 = clock64();
        while (clock64() - t0 < 4000000) {}
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();               // neither CTA leaves while the other may still signal it
    if (warp == 1) {
        if (PAIR) tmem_dealloc_pair(tmem, 512);
        else tmem_dealloc(tmem, 512);
    }
}

// ------------------------------------------------------------------------------------------------ host side
static bool ns_attributes() {
    static PerDeviceFlag attr_set;
    if (attr_set.get()) return true;
    if (cudaFuncSetAttribute(ns_kernel<NS_ALONE>, cudaFuncAttributeMaxDynamicSharedMemorySize, NS_SMEM_ALL) != cudaSuccess ||
        cudaFuncSetAttribute(ns_kernel<NS_SHARE>, cudaFuncAttributeMaxDynamicSharedMemorySize, NS_SMEM_ALL) != cudaSuccess ||
        cudaFuncSetAttribute(ns_kernel<NS_PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize, NS_SMEM_ALL) != cudaSuccess ||
        cudaFuncSetAttribute(ns_kernel<NS_ALONE>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
        cudaFuncSetAttribute(ns_kernel<NS_SHARE>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
        (void)cudaGetLastError();
        return false;
    }
    attr_set.set();
    return true;
}

struct NsPlan {
    NsParams p;
    size_t hi0, hi1, lo, H[3], L[2], W[3], D[3], part, norm, arrived, total;
    int norm_blocks;
};

static int ns_tri_tiles(int n, int tr, int nt) {
    int t = 0;
    for (int i = 0; i < (n + tr - 1) / tr; ++i) t += ns_tri_row(i, n, tr, nt);
    return t;
}

// Clusters of 2, 4, 8 or 16 CTAs the device holds at a time, with all of an SM's shared memory to a CTA; `pair`: of the kernel for CTA pairs.
static int ns_clusters(int ctas, bool pair = false) {
    static std::atomic<int> known[64][5];
    int k = 0;
    while ((2 << k) < ctas) ++k;
    std::atomic<int>& slot = known[PerDeviceFlag::dev()][pair ? 4 : k];
    int n = slot.load(std::memory_order_relaxed);
    if (n) return n - 1;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.gridDim = dim3(ctas); cfg.blockDim = dim3(NS_THREADS); cfg.dynamicSmemBytes = NS_SMEM_ALL; cfg.attrs = attr; cfg.numAttrs = 1;
    if (!ns_attributes() || cudaOccupancyMaxActiveClusters(&n, pair ? ns_kernel<NS_PAIR> : ns_kernel<NS_SHARE>, &cfg) != cudaSuccess || n < 0) {
        (void)cudaGetLastError();
        n = 0;
    }
    slot.store(n + 1, std::memory_order_relaxed);
    return n;
}

static NsPlan ns_plan(int batch, int rows, int cols) {
    NsPlan l = {};
    NsParams& p = l.p;
    const int sms = num_sms();
    p.batch = batch;
    p.in.rows = rows; p.in.cols = cols; p.in.tall = rows > cols;
    p.n = std::min(rows, cols); p.m = std::max(rows, cols);
    p.ldx = (p.m + 63) / 64 * 64; p.lda = (p.n + 63) / 64 * 64;
    p.terms = p.n <= 64 ? 3 : 1;
    // CTAs per matrix: what the widest phase can use with its narrowest tiles, at most all SMs
    const int batch1 = batch < 1 ? 1 : batch;
    const int rows128 = (p.n + 127) / 128, rows256 = (p.n + 255) / 256;
    auto across = [](int width, int nt) { return (width + nt - 1) / nt; };
    int g = std::min({std::max(rows128 * across(p.m, 64), 1), sms, std::max(1, sms / batch1)});
    // As a cluster (of a power of two) where the device holds one for every matrix at a time: as nine clusters of 16 that take turns, 9 x 144 x
    // 816 took 211 us, as nine groups of a cooperative launch 120.  And where that leaves few CTAs unused: 20 x 144 x 816 in clusters of 4
    // took 202 us, in groups of 7 140; 12 x 160 x 160 with 8 and 12 125 and 99 us.
    int q = 1;
    while (q * 2 <= g) q *= 2;
    if (q > 1 && g <= 16 && 4 * q >= 3 * g && ns_clusters(q) >= std::min(batch1, sms / q)) {
        g = q;
        p.cluster = 1;
    }
    p.G = g;
    p.groups = std::min(batch1, std::max(1, sms / g));
    // Cycles of a phase, by a model that ranks the choices below: its start, rounds of tiles over the group's CTAs, and the last tile's drain.  A round takes the longer of
    // its slices and the drain of the tile before it; a 64-deep slice the longest of its MMAs, the issuing threads' hand-over (one of
    // two threads, or a pair's only one) and its operands' way out of L2 (7000 bytes a cycle for all SMs).
    auto cost = [&](int tiles, int chunks, int nt, bool pair) {
        const int units = pair ? g / 2 : g, rounds = (tiles + units - 1) / units, busy = std::min(tiles, units) * (pair ? 2 : 1);
        const long long bytes = NS_CHUNK + (pair ? nt / 2 : nt) * 128, drain = 60 * nt;
        const long long slice = std::max<long long>({pair ? 700 : 330, 2 * std::max(nt, 128), p.groups * busy * bytes / 7000});
        return 2500 + rounds * std::max(chunks * slice, drain) + drain;
    };
    constexpr long long BARRIER = 2500, SPLIT = 10000;          // a barrier; what splitting A adds: parts written, barrier, parts summed
    const int cm = (p.m + 63) / 64, cn = (p.n + 63) / 64;
    struct Choice { long long a, s, x; int nt_a, nt_s, nt_x, tiles_a, tiles_s, tiles_x, full_a, full_s, splits, share; };
    auto choose = [&](bool pair) {
        Choice c = {};
        const int rows = pair ? rows256 : rows128, tr = pair ? 256 : 128, wide = pair ? 256 : 128, narrow = wide / 2;
        c.x = c.s = c.a = -1;
        for (int nt : {wide, narrow}) {
            const int all_x = rows * across(p.m, nt), all_n = rows * across(p.n, nt), tri = ns_tri_tiles(p.n, tr, nt);
            auto take = [](long long& best, long long now) { const bool better = best < 0 || now < best; if (better) best = now; return better; };
            if (take(c.x, cost(all_x, cn, nt, pair))) { c.nt_x = nt; c.tiles_x = all_x; }
            // all tiles of a symmetric product where the group has a CTA for each (no mirrored stores), otherwise those of the lower triangle
            const bool full = !pair && all_n <= g;
            if ((full || nt == wide || pair) && take(c.s, cost(full ? all_n : tri, cn, nt, pair))) { c.nt_s = nt; c.full_s = full; c.tiles_s = full ? all_n : tri; }
            if (full && take(c.a, cost(all_n, cm, nt, pair))) { c.nt_a = nt; c.full_a = 1; c.tiles_a = all_n; c.splits = c.share = 1; }
            // Few tiles: a cluster's CTAs share each, a range of the long axis a CTA (one SM's operands arrive at 70 bytes a cycle, whatever the
            // others do: 512 x 2048 129.5 -> 119.5 us, 256 x 2304 123 -> 107 us, but 1000 x 2048, which fills the SMs, 174 -> 191 us).  A CTA drains
            // its share of the columns; the exchange is a cluster barrier and the columns' way.
            for (int k = 2; !pair && k <= 4; k *= 2) {
                if (!full || all_n * k > g || g % k || cm < 2 * k || (!p.cluster && ns_clusters(k) * k < p.groups * g)) continue;
                if (take(c.a, cost(all_n * k, (cm + k - 1) / k, nt, false) - 60 * nt * (k - 1) / k + 1500 + 32 * nt)) { c.nt_a = nt; c.full_a = 1; c.tiles_a = all_n; c.splits = 1; c.share = k; }
            }
            if (nt == wide || pair) {
                // or the lower triangle with the long axis split over the CTAs, whose parts meet after another barrier
                const int s = pair ? 1 : std::max(1, std::min(g / tri, cm / 4));
                if (take(c.a, cost(tri * s, (cm + s - 1) / s, nt, pair) + (s > 1 ? SPLIT : 0))) { c.nt_a = nt; c.full_a = 0; c.tiles_a = tri; c.splits = s; c.share = 1; }
            }
        }
        return c;
    };
    Choice c = choose(false);
    // Pairs meet at grid barriers: only where the device holds all of them at a time.
    if (g == sms && sms % 2 == 0 && p.n > 128 && 2 * ns_clusters(2, true) >= sms) {
        const Choice two = choose(true);
        if (two.a + two.s + two.x < c.a + c.s + c.x) { c = two; p.pair = 1; }
    }
    p.tr = p.pair ? 256 : 128;
    p.nt_a = c.nt_a; p.nt_s = c.nt_s; p.nt_x = c.nt_x;
    p.tiles_a = c.tiles_a; p.tiles_s = c.tiles_s; p.tiles_x = c.tiles_x;
    p.full_a = c.full_a; p.full_s = c.full_s; p.splits = c.splits; p.share = c.share;
    p.stage_bytes = ns_depth(p.pair) * (NS_CHUNK + std::max(p.nt_x, std::max(p.nt_s, p.nt_a)) * (p.pair ? 64 : 128));
    p.stages = std::min(NS_STAGES, (NS_SMEM - (p.share > 1 ? p.nt_a * 512 : 0)) / p.stage_bytes);
    // Two steps of X at a time save one A and one X product of every two and cost three more n x n products, and a barrier each.  Taken where
    // the model's saving is 7/5 of its cost, since it errs (saving over cost, one and two steps at a time, five steps in all):
    //   512 x 2048 0.68 119 142 us, 1000 x 2048 0.95 176 193, 4096 x 4096 0.94 1497 1642, 512 x 4608 1.04 166 172, 2048 x 4608 1.22 504 496,
    //   300 x 9000 1.33 168 173, 1024 x 4608 1.45 243 238, 512 x 8192 1.47 201 201, 512 x 13200 1.74 250 233, 4096 x 9216 1.82 2664 2379,
    //   2048 x 8192 2.02 819 691, 640 x 20800 2.75 398 340, 40 x 130 x 4200 3.72 805 627.
    // Rounding errors of A' are of A's size, not of its small entries': fine for one such step (up to twice the error of O on spectra over
    // several decades: 1.3e-3 at 512 x 13200 against 7e-4 at 512 x 2048), not for a chain of them.
    p.merge = p.terms == 1 && 5 * (c.a + c.x + 2 * BARRIER) > 7 * 3 * (c.s + BARRIER);
    l.norm_blocks = (int)std::min<size_t>(NS_NORM_BLOCKS, ((size_t)rows * cols + 2047) / 2048);
    p.n_norm = p.cluster || g == 1 ? g : l.norm_blocks;
    size_t at = 0;
    auto take = [&](size_t& where, size_t bytes) { where = at; at += (bytes + 255) / 256 * 256; };
    const size_t x = (size_t)p.groups * p.n * p.ldx * 2, a = (size_t)p.groups * p.n * p.lda * 2;
    take(l.hi0, x); take(l.hi1, x); take(l.lo, x);
    for (int k = 0; k < 3; ++k) {
        take(l.H[k], k < 2 || p.merge ? a : 0);
        take(l.W[k], k == 0 || p.merge ? 2 * a : 0);
        take(l.D[k], (size_t)p.groups * p.lda * 4);
        if (k < 2) take(l.L[k], p.terms == 3 ? a : 0);
    }
    take(l.part, p.splits > 1 ? (size_t)p.groups * p.splits * p.tiles_a * p.nt_a * 128 * 4 : 0);
    take(l.norm, (size_t)(p.cluster || g == 1 ? p.groups : batch1) * p.n_norm * 8);
    take(l.arrived, (size_t)p.groups * 4);
    l.total = at;
    return l;
}

static int ns_map(CUtensorMap* map, const void* ptr, int rows, int ld, int groups, int box_rows, int box_chunks) {
    const cuuint64_t dims[4] = {64, (cuuint64_t)rows, (cuuint64_t)(ld / 64), (cuuint64_t)groups};
    const cuuint64_t strides[3] = {(cuuint64_t)ld * 2, 128, (cuuint64_t)rows * ld * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, (cuuint32_t)box_chunks, 1};
    return tmap_tiled(map, 4, ptr, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

static int ns_check(int batch, int rows, int cols, int steps, const float* coef, float eps) {
    if (batch < 0 || rows <= 0 || cols <= 0 || steps < 1 || !(eps >= 0.f)) return DR_ERR_INVALID_ARG;
    if (rows > DR_NS_MAX_DIM || cols > DR_NS_MAX_DIM || steps > DR_NS_MAX_STEPS || batch > 65535) return DR_ERR_UNSUPPORTED;
    if (coef)
        for (int i = 0; i < 3 * steps; ++i)
            if (!std::isfinite(coef[i])) return DR_ERR_INVALID_ARG;
    return DR_OK;
}

static int ns_run(int batch, NsInput in, int steps, const float* coef, char* ws, size_t ws_bytes, cudaStream_t s) {
    in.tall = in.rows > in.cols;
    in.vec = (in.cols & 7) == 0 && aligned16(in.g) && aligned16(in.v) && aligned16(in.w) && aligned16(in.out);
    float own[3 * DR_NS_MAX_STEPS];
    const float usual[3] = {3.4445f, -4.7750f, 2.0315f};
    for (int i = 0; i < 3 * steps; ++i) own[i] = coef ? coef[i] : usual[i % 3];
    const NsSmallPlan small = ns_small_plan(batch, in.rows, in.cols);
    if (small.ctas) {
        if (ws_bytes < small.bytes) return DR_ERR_WORKSPACE;
        return batch == 0 ? DR_OK : ns_small_run(small, batch, in, steps, own, ws, s);
    }
    NsPlan l = ns_plan(batch, in.rows, in.cols);
    if (ws_bytes < l.total) return DR_ERR_WORKSPACE;
    if (batch == 0) return DR_OK;
    NsParams& p = l.p;
    p.in = in;
    p.steps = steps;
    for (int i = 0; i < 3 * steps; ++i) p.coef[i] = own[i];
    p.hi[0] = (__half*)(ws + l.hi0); p.hi[1] = (__half*)(ws + l.hi1); p.lo = (__half*)(ws + l.lo);
    for (int k = 0; k < 3; ++k) {
        p.H[k] = (__half*)(ws + l.H[k]); p.W[k] = (float*)(ws + l.W[k]); p.D[k] = (float*)(ws + l.D[k]);
        if (k < 2) p.L[k] = (__half*)(ws + l.L[k]);
    }
    p.part = (float*)(ws + l.part);
    p.norm = (double*)(ws + l.norm); p.arrived = (unsigned*)(ws + l.arrived);
    p.status = dev_status_ptr();
    alignas(64) NsMaps maps;
    int st = DR_OK;
    auto put = [&](CUtensorMap& m, const void* ptr, int ld, int box_rows, int box_chunks) {
        if (st == DR_OK) st = ns_map(&m, ptr, p.n, ld, p.groups, box_rows, box_chunks);
    };
    auto same = [](CUtensorMap& m, const CUtensorMap& o) { std::memcpy(&m, &o, sizeof(m)); };
    const bool lows = p.terms == 3;
    const int depth = ns_depth(p.pair), narrow = p.pair ? 128 : 64;
    for (int k = 0; k < 2; ++k) {
        put(maps.hi[k], p.hi[k], p.ldx, 128, depth);
        if (p.nt_a == narrow) put(maps.ba_hi[k], p.hi[k], p.ldx, 64, depth); else same(maps.ba_hi[k], maps.hi[k]);
        put(maps.bx_hi[k], p.hi[k], p.ldx, 64 * depth, p.nt_x == narrow ? 1 : 2);
    }
    for (int k = 0; k < 3; ++k) {
        if (k == 2 && !p.merge) {               // not read
            same(maps.H[2], maps.H[0]);
            same(maps.bs[2], maps.bs[0]);
            break;
        }
        put(maps.H[k], p.H[k], p.lda, 128, depth);
        if (p.nt_s == narrow) put(maps.bs[k], p.H[k], p.lda, 64, depth); else same(maps.bs[k], maps.H[k]);
    }
    if (lows) {
        put(maps.lo, p.lo, p.ldx, 128, 2);
        put(maps.L[0], p.L[0], p.lda, 128, 2);
        put(maps.L[1], p.L[1], p.lda, 128, 2);
        if (p.nt_a == 64) put(maps.ba_lo, p.lo, p.ldx, 64, 2); else same(maps.ba_lo, maps.lo);
        if (p.nt_x == 64) put(maps.bx_lo, p.lo, p.ldx, 128, 1); else same(maps.bx_lo, maps.lo);
        if (p.nt_s == 64) put(maps.bs_lo, p.L[0], p.lda, 64, 2); else same(maps.bs_lo, maps.L[0]);
    } else {                                    // not read
        for (CUtensorMap* m : {&maps.lo, &maps.L[0], &maps.L[1], &maps.ba_lo, &maps.bx_lo, &maps.bs_lo}) same(*m, maps.H[0]);
    }
    if (st != DR_OK) return st;
    if (!ns_attributes()) return DR_ERR_CUDA;
    const bool counted = !(p.cluster || p.G == 1);
    if (counted) {
        ns_begin_kernel<<<dim3((unsigned)p.n_norm, (unsigned)p.batch), 256, 0, s>>>(p.in, p.norm, p.arrived, p.groups);
        count_launch();
        st = launch_status();
        if (st != DR_OK) return st;
    }
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3((unsigned)(p.groups * p.G)); cfg.blockDim = dim3(NS_THREADS); cfg.dynamicSmemBytes = NS_SMEM_ALL; cfg.stream = s;
    cfg.attrs = attr;
    if (counted) {
        attr[0].id = cudaLaunchAttributeCooperative;
        attr[0].val.cooperative = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = p.pair ? 2 : p.share; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = p.pair || p.share > 1 ? 2 : 1;
    } else if (p.cluster) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = p.G; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.numAttrs = 1;
    }
    if (cudaLaunchKernelEx(&cfg, p.pair ? ns_kernel<NS_PAIR> : p.share > 1 ? ns_kernel<NS_SHARE> : ns_kernel<NS_ALONE>, maps, p) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
    count_launch();
    return launch_status();
}

// One of the kernels on two CTAs without the cluster that its parameters name.  (The kernel of CTA pairs is not among them: the driver refuses
// to launch it so.)
static int ns_lost_cluster(int kind, cudaStream_t stream) {
    if (kind == 0) return ns_small_lost_cluster(stream);
    NsMaps maps = {};
    NsParams p = {};
    p.G = 2;
    p.share = 2;
    p.cluster = kind == 1;
    p.status = dev_status_ptr();
    if (!ns_attributes()) return DR_ERR_CUDA;
    (kind == 1 ? ns_kernel<NS_ALONE> : ns_kernel<NS_SHARE>)<<<2, NS_THREADS, NS_SMEM_ALL, stream>>>(maps, p);
    count_launch();
    return launch_status();
}

}  // namespace dr

using namespace dr;

extern "C" int dr_selftest_lost_cluster(int kind, void* stream) {
    if (kind < 0 || kind > 2) return DR_ERR_INVALID_ARG;
    return dev_status_ptr() ? ns_lost_cluster(kind, (cudaStream_t)stream) : DR_ERR_CUDA;
}

extern "C" int dr_orthogonalise_workspace_bytes(int batch, int rows, int cols, size_t* bytes) {
    if (!bytes) return DR_ERR_INVALID_ARG;
    const int st = ns_check(batch, rows, cols, 1, nullptr, 0.f);
    if (st != DR_OK) return st;
    const NsSmallPlan small = ns_small_plan(batch, rows, cols);
    *bytes = small.ctas ? small.bytes : ns_plan(batch, rows, cols).total;
    return DR_OK;
}

extern "C" int dr_orthogonalise_plan(int batch, int rows, int cols, int plan[8]) {
    if (!plan) return DR_ERR_INVALID_ARG;
    const int st = ns_check(batch, rows, cols, 1, nullptr, 0.f);
    if (st != DR_OK) return st;
    const NsSmallPlan small = ns_small_plan(batch, rows, cols);
    for (int i = 0; i < 8; ++i) plan[i] = 0;
    if (small.ctas) {
        plan[0] = DR_NS_KERNEL_SMALL; plan[1] = small.ctas; plan[2] = small.groups; plan[4] = plan[5] = 1; plan[6] = small.terms; plan[7] = small.ctas > 1;
        return DR_OK;
    }
    const NsParams p = ns_plan(batch, rows, cols).p;
    plan[0] = p.pair ? DR_NS_KERNEL_PAIR : p.share > 1 ? DR_NS_KERNEL_SHARE : DR_NS_KERNEL_ALONE;
    plan[1] = p.G; plan[2] = p.groups; plan[3] = p.merge; plan[4] = p.splits; plan[5] = p.share; plan[6] = p.terms; plan[7] = p.cluster;
    return DR_OK;
}

extern "C" int dr_orthogonalise(int batch, int rows, int cols, const void* g, int steps, const float* coef, float eps, void* o, void* workspace,
                                size_t workspace_bytes, unsigned flags, void* stream) {
    const int st = ns_check(batch, rows, cols, steps, coef, eps);
    if (st != DR_OK) return st;
    if (!g || !o || !workspace || (flags & ~(unsigned)DR_NS_G_F32)) return DR_ERR_INVALID_ARG;
    const bool f32 = flags & DR_NS_G_F32;
    if (((uintptr_t)g & (f32 ? 3u : 1u)) || ((uintptr_t)o & 1u) || ((uintptr_t)workspace & 255)) return DR_ERR_ALIGNMENT;
    NsInput in = {};
    in.rows = rows; in.cols = cols; in.g = g; in.g_f32 = f32; in.eps = eps; in.out = (__nv_bfloat16*)o;
    return ns_run(batch, in, steps, coef, (char*)workspace, workspace_bytes, (cudaStream_t)stream);
}

extern "C" int dr_muon_update(int batch, int rows, int cols, float* w, float* v, const float* g, float lr, float momentum, float decay, int nesterov,
                              int steps, const float* coef, float eps, void* w_bf16, void* workspace, size_t workspace_bytes, void* stream) {
    const int st = ns_check(batch, rows, cols, steps, coef, eps);
    if (st != DR_OK) return st;
    if (!w || !v || !g || !workspace) return DR_ERR_INVALID_ARG;
    if (((uintptr_t)w & 3u) || ((uintptr_t)v & 3u) || ((uintptr_t)g & 3u) || ((uintptr_t)w_bf16 & 1u) || ((uintptr_t)workspace & 255)) return DR_ERR_ALIGNMENT;
    NsInput in = {};
    in.rows = rows; in.cols = cols; in.g = g; in.g_f32 = 1; in.eps = eps; in.v = v; in.w = w; in.momentum = momentum; in.nesterov = nesterov != 0;
    in.lr_scale = lr * (rows > cols ? sqrtf((float)rows / (float)cols) : 1.f);
    in.keep = 1.f - lr * decay;
    in.out = (__nv_bfloat16*)w_bf16;
    return ns_run(batch, in, steps, coef, (char*)workspace, workspace_bytes, (cudaStream_t)stream);
}
