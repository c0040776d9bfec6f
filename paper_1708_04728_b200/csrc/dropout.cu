// Dropout: y = residual + keep * x / (1 - p), the mask drawn by a counter-based generator (dropout.cuh) and never stored; the backward
// pass is the same call on the gradient.
// Bound by memory where rows allow 16-byte accesses (200704 x 256 bfloat16 with residual 59 us, 5.2 TB/s, 0.79 of a plain copy's rate), by issue slots
// elsewhere (50176 x 333 float32 in rows of 357 36 us, 70 % of the slots busy).
#include <algorithm>
#include <climits>

#include "common.cuh"
#include "dropout.cuh"

namespace dr {

struct DropParams {
    unsigned long long n;       // items: vectors of 8 elements, or elements
    unsigned long long tail;    // elements behind the last whole vector (dense tensors)
    int C, ldx, ldr, ldy;
    int cv;                     // vectors of a row
    int step_row, step_col;     // what a walk over all threads adds to a row and a place in it
    uint32_t magic;             // 2^32 / C, rounded up, where C < 256
    const void *x, *r;
    void* y;
    DropKey key;
};

template <typename T> __device__ __forceinline__ float drop_ld(const void* p, size_t i);
template <> __device__ __forceinline__ float drop_ld<float>(const void* p, size_t i) { return __ldcs((const float*)p + i); }
template <> __device__ __forceinline__ float drop_ld<__nv_bfloat16>(const void* p, size_t i) {
    const unsigned short u = __ldcs((const unsigned short*)p + i);
    return __uint_as_float((uint32_t)u << 16);
}
__device__ __forceinline__ void drop_st(float* p, float v) { *p = v; }
__device__ __forceinline__ void drop_st(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// eight neighbours as they lie in memory
template <typename T> struct Vec8;
template <> struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = __ldcs((const float4*)p); b = __ldcs((const float4*)p + 1); }
    __device__ __forceinline__ float get(int i) const { const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}; return v[i]; }
    static __device__ __forceinline__ void store(float* p, const float* v) {
        ((float4*)p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        ((float4*)p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
};
template <> struct Vec8<__nv_bfloat16> {
    uint4 a;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = __ldcs((const uint4*)p); }
    __device__ __forceinline__ float get(int i) const { const uint32_t v[4] = {a.x, a.y, a.z, a.w}; return (i & 1) ? bf16_hi(v[i >> 1]) : bf16_lo(v[i >> 1]); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* v) {
        *(uint4*)p = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
    }
};

// Rows of a multiple of 8 channels on 16-byte boundaries, or dense tensors of any shape taken as one row: a vector of 8 is a counter of the
// generator.  A thread has the loads of AHEAD vectors in flight while it draws their masks.
constexpr int DROP_AHEAD = 4;
template <typename TX, typename TY, bool RES, bool DENSE>
__global__ void __launch_bounds__(256) dropout_vec_kernel(const DropParams p) {
    const unsigned long long off = drop_offset(p.key);
    const unsigned long long stride = (unsigned long long)gridDim.x * 256;
    unsigned long long i = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
    size_t row = 0;
    int col = 0;
    if (!DENSE) { row = i / p.cv; col = (int)(i - row * p.cv); }
    auto place = [&](size_t ld) { return DENSE ? (size_t)i * 8 : row * ld + (size_t)col * 8; };
    auto next = [&]() {
        i += stride;
        if (!DENSE) {
            row += p.step_row;
            col += p.step_col;
            if (col >= p.cv) { col -= p.cv; ++row; }
        }
    };
    while (i < p.n) {
        Vec8<TX> x[DROP_AHEAD];
        Vec8<TY> r[DROP_AHEAD];
        size_t at[DROP_AHEAD];
        unsigned long long counter[DROP_AHEAD];
#pragma unroll
        for (int k = 0; k < DROP_AHEAD; ++k) {
            counter[k] = i;
            if (i < p.n) {
                at[k] = place(p.ldy);
                x[k].load((const TX*)p.x + place(p.ldx));
                if (RES) r[k].load((const TY*)p.r + place(p.ldr));
            }
            next();
        }
#pragma unroll
        for (int k = 0; k < DROP_AHEAD; ++k) {
            if (counter[k] >= p.n) break;
            const uint4 w = drop_words(p.key, off, counter[k]);
            float v[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                v[c] = drop_keep(w, c, p.key.thr) ? x[k].get(c) * p.key.scale : 0.f;
                if (RES) v[c] += r[k].get(c);
            }
            Vec8<TY>::store((TY*)p.y + at[k], v);
        }
    }
    if (DENSE && blockIdx.x == 0 && threadIdx.x < p.tail) {
        const size_t e = (size_t)p.n * 8 + threadIdx.x;
        const float v = drop_keep_at(p.key, off, e) ? drop_ld<TX>(p.x, e) * p.key.scale : 0.f;
        drop_st((TY*)p.y + e, RES ? drop_ld<TY>(p.r, e) + v : v);
    }
}

// Any other rows: a warp takes 256 neighbouring elements.  Each lane draws a vector's mask, and gets the bits of the elements it moves (lane, lane + 32,
// ...: whole lines of memory) from the lanes that drew them.
// The issue slots bound it, so places are 32 bits from the row's start, and a row of 256 or more elements (NARROW false) ends at most once in them.
template <typename TX, typename TY, bool RES, bool NARROW>
__global__ void __launch_bounds__(256) dropout_any_kernel(const DropParams p) {
    const unsigned long long off = drop_offset(p.key);
    const int lane = threadIdx.x & 31;
    const unsigned long long stride = (unsigned long long)gridDim.x * 8 * 256;
    unsigned long long e = ((unsigned long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * 256;
    size_t row = e / p.C;
    int col = (int)(e - row * p.C);
    const uint32_t C = (uint32_t)p.C, gap_x = (uint32_t)(p.ldx - p.C), gap_r = (uint32_t)(p.ldr - p.C), gap_y = (uint32_t)(p.ldy - p.C);
    for (; e < p.n; e += stride) {
        const TX* const x0 = (const TX*)p.x + row * p.ldx;
        const TY* const r0 = (const TY*)p.r + (RES ? row * p.ldr : 0);
        TY* const y0 = (TY*)p.y + row * p.ldy;
        const uint32_t left = (uint32_t)min(p.n - e, 256ull), first = (uint32_t)col + lane;
        // rows passed by the element `i` of the row on: what the gaps between rows count for
        auto passed = [&](uint32_t i) { return NARROW ? (C == 1 ? i : __umulhi(i, p.magic)) : (i >= C ? 1u : 0u); };
        auto place = [](uint32_t i, uint32_t over, uint32_t gap) { return NARROW ? i + (size_t)over * gap : (size_t)(over ? i + gap : i); };
        float x[8], r[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t i = first + 32 * k, over = passed(i);
            if (32 * k + lane < left) {
                x[k] = drop_ld<TX>(x0, place(i, over, gap_x));
                if (RES) r[k] = drop_ld<TY>(r0, place(i, over, gap_r));
            }
        }
        const uint4 w = drop_words(p.key, off, (e >> 3) + lane);
        uint32_t bits = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) bits |= drop_keep(w, c, p.key.thr) ? 1u << c : 0u;
        const uint32_t mine = 1u << (lane & 7);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t i = first + 32 * k, over = passed(i);
            const uint32_t b = __shfl_sync(0xffffffffu, bits, 4 * k + (lane >> 3)) & mine;
            const float v = b ? x[k] * p.key.scale : 0.f;
            if (32 * k + lane < left) drop_st(y0 + place(i, over, gap_y), RES ? r[k] + v : v);
        }
        row += p.step_row;
        col += p.step_col;
        if (col >= p.C) { col -= p.C; ++row; }
    }
}

template <typename TX, typename TY, bool RES>
static void drop_launch(DropParams p, cudaStream_t s) {
    const int xs = 16 / sizeof(TX), ys = 16 / sizeof(TY);       // elements of 16 bytes
    const bool dense = p.ldx == p.C && p.ldy == p.C && (!RES || p.ldr == p.C);
    const bool aligned = aligned16(p.x) && aligned16(p.y) && aligned16(p.r);
    const bool rows = p.C % 8 == 0 && p.ldx % xs == 0 && p.ldy % ys == 0 && (!RES || p.ldr % ys == 0);
    const unsigned long long most = (unsigned long long)num_sms() * 8;
    if (aligned && (dense || rows)) {
        p.tail = p.n % 8;
        p.n /= 8;
        p.cv = p.C / 8;
        unsigned long long blocks = (p.n + 255) / 256;
        if (blocks > most) blocks = std::min(most, (p.n + 256 * DROP_AHEAD - 1) / (256 * DROP_AHEAD));
        const unsigned grid = (unsigned)std::max(1ull, blocks);
        if (!dense) { p.step_row = (int)(grid * 256ull / p.cv); p.step_col = (int)(grid * 256ull % p.cv); }
        if (dense) dropout_vec_kernel<TX, TY, RES, true><<<grid, 256, 0, s>>>(p);
        else dropout_vec_kernel<TX, TY, RES, false><<<grid, 256, 0, s>>>(p);
    } else {
        const unsigned grid = (unsigned)std::min(most, (p.n + 2047) / 2048);
        p.step_row = (int)(grid * 2048ull / p.C);
        p.step_col = (int)(grid * 2048ull % p.C);
        p.magic = p.C > 1 && p.C < 256 ? (uint32_t)((0x100000000ull + p.C - 1) / p.C) : 0u;
        if (p.C < 256) dropout_any_kernel<TX, TY, RES, true><<<grid, 256, 0, s>>>(p);
        else dropout_any_kernel<TX, TY, RES, false><<<grid, 256, 0, s>>>(p);
    }
}
template <typename TX, typename TY>
static void drop_launch(const DropParams& p, cudaStream_t s) {
    if (p.r) drop_launch<TX, TY, true>(p, s);
    else drop_launch<TX, TY, false>(p, s);
}

static bool type_aligned(const void* p, size_t size) { return ((uintptr_t)p & (size - 1)) == 0; }

}  // namespace dr

using namespace dr;

extern "C" int dr_dropout(size_t rows, int C, const void* x, int ldx, const void* residual, int ldr, void* y, int ldy, double p, unsigned long long seed,
                          unsigned long long offset, const unsigned long long* step, unsigned flags, void* stream) {
    if (C <= 0 || (flags & ~(DR_DROP_X_F32 | DR_DROP_Y_F32)) || !drop_p_ok(p)) return DR_ERR_INVALID_ARG;
    if (!ldx) ldx = C;
    if (!ldr) ldr = C;
    if (!ldy) ldy = C;
    if (ldx < C || ldr < C || ldy < C || rows > (size_t)LLONG_MAX / 16 / C) return DR_ERR_INVALID_ARG;
    if (rows == 0) return DR_OK;
    if (!x || !y) return DR_ERR_INVALID_ARG;
    const bool xf = flags & DR_DROP_X_F32, yf = flags & DR_DROP_Y_F32;
    if (!type_aligned(x, xf ? 4 : 2) || !type_aligned(y, yf ? 4 : 2) || !type_aligned(residual, yf ? 4 : 2) || !type_aligned(step, 8)) return DR_ERR_ALIGNMENT;
    DropParams q = {};
    q.n = (unsigned long long)rows * C;
    q.C = C; q.ldx = ldx; q.ldr = ldr; q.ldy = ldy;
    q.x = x; q.r = residual; q.y = y;
    q.key = drop_key(p, seed, offset, step);
    const cudaStream_t s = (cudaStream_t)stream;
    if (xf && yf) drop_launch<float, float>(q, s);
    else if (xf) drop_launch<float, __nv_bfloat16>(q, s);
    else if (yf) drop_launch<__nv_bfloat16, float>(q, s);
    else drop_launch<__nv_bfloat16, __nv_bfloat16>(q, s);
    count_launch();
    return launch_status();
}
