// Layer normalisation over the channels of a pixel, forward and backward:
//   y = (x - mean) * rstd * gamma + beta,   mean, var over the C channels of a row, rstd = 1 / sqrt(var + eps)
//   t = dy * gamma,  xhat = (x - mean) * rstd,
//   dx = rstd * (t - mean_c(t) - xhat * mean_c(t * xhat)),   dgamma = sum_rows dy * xhat,   dbeta = sum_rows dy
//
// Both passes are bound by memory: a row is read once into registers, its statistics are taken there (the mean first,
// then the squared distances from it: no cancellation), and the result is written.  A team of TW threads (8 .. 512)
// owns a row; teams walk the rows with a fixed stride, keep gamma, beta and their sums of the weight gradients in
// registers, and have the next rows' loads in flight while they work on this one.
//
// Measured on a B200 against a copy of 1 Gi elements at 6530 GB/s.  200704 rows x 256 channels, bfloat16: forward 38 us
// (5.4 TB/s, 0.83 of that copy; a copy of these 206 MB takes 35 us), backward 57 us (5.4 TB/s, 0.83); with loads straight into
// registers, one row ahead, they took 90 and 241 us.  12544 x 2048, float32 x and dx: backward 48 us (5.4 TB/s, 0.82).
// 50176 x 333 inside rows of 501 (no row but every eighth aligned): forward 16 us (4.1 TB/s), backward 35 us.  Neither memory
// (29 % in the forward pass) nor the issue slots (47 %) are full: latency, with 114 registers a thread and so 16 warps on an
// SM.  Of the 207 kernels here 32 of the backward pass spill 4 .. 36 bytes at 128 registers, all phased ones of 16 channels a
// thread among them, and one of the forward pass 4.  49 x 1024: 5.5 and 8.3 us, the launches (a kernel that does nothing
// takes 2 us between its neighbours; the backward pass has two).
#include <algorithm>
#include <initializer_list>
#include <map>
#include <mutex>
#include <tuple>

#include "common.cuh"
#include "umma_ptx.cuh"

namespace dr {

struct LnParams {
    size_t M;
    int C, ldx, ldy, lddx;      // ldy is dy's in the backward pass
    const void *x, *dy;
    void *y, *dx;
    const float *gamma, *beta, *mean_in, *rstd_in;
    float *mean, *rstd;
    float eps, inv_c;
    float* partials;            // [n_part][2][C]: one row of sums per block, or nullptr
    int n_part;
    float *dgamma, *dbeta;
};

// How a row lies in memory, in vectors of 8 elements where all tensors are bfloat16 and of 4 where one is float32 (16 bytes of the widest
// type).  ALIGNED: every row of every tensor is a whole number of vectors from a vector's boundary on.
// PHASED: rows start anywhere, but all tensors are off the boundary by the same number of elements in any one row, and a
// team takes rows a multiple of 8 apart, so that its offset never changes: whole vectors from the first boundary on, and
// the few channels in front of it and behind the last vector one to a thread.  SINGLE: neither; single elements.
enum { LN_ALIGNED, LN_PHASED, LN_SINGLE };

constexpr int LN_BWD_THREADS = 512;
constexpr size_t LN_SMEM_MAX = 216 * 1024;
// Rows a thread has on their way besides the one it works on (ALIGNED and PHASED: copied to shared memory by cp.async, each thread
// its own vectors, so that no barrier is needed): 24 KB or more in flight per SM at all times.
__host__ __device__ constexpr int ln_ring(int bytes_per_row) { return bytes_per_row <= 96 ? 4 : 3; }

// Two float32 operations in one instruction.
__device__ __forceinline__ float2 f2_add(float2 a, float2 b) {
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(d)) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return d;
}
__device__ __forceinline__ float2 f2_mul(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(d)) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
    return d;
}
__device__ __forceinline__ float2 f2_fma(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<unsigned long long&>(d)) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
    return d;
}
__device__ __forceinline__ float2 f2(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2& f2_at(float* v, int i) { return reinterpret_cast<float2*>(v)[i]; }

template <int B> __device__ __forceinline__ void cp_async(uint32_t dst, const void* src, bool in) {       // zeros where !in
    if (B == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
    else if (B == 4) asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(in ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// E consecutive channels of a row as they lie in memory.  E = 8: 16 bytes of bfloat16; E = 4, where one of the tensors is
// float32: 16 bytes of that one (a warp's access must cover whole 32-byte sectors, or they are fetched twice); E = 1.
__device__ __forceinline__ float ln_value(float v) { return v; }
__device__ __forceinline__ float ln_value(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void ln_store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void ln_store1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
template <int E> __device__ __forceinline__ void ln_store(__nv_bfloat16* p, const float* v) {
    if (E == 8) *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4 % E], v[5 % E]), pack_bf16(v[6 % E], v[7 % E]));
    else if (E == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16(v[0], v[1 % E]), pack_bf16(v[2 % E], v[3 % E]));
    else ln_store1(p, v[0]);
}
template <int E> __device__ __forceinline__ void ln_store(float* p, const float* v) {
    if (E == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1 % E], v[2 % E], v[3 % E]);
    else ln_store1(p, v[0]);
}

// Sum over the team's threads of N values, the same bits in every thread.  Teams of more than a warp meet at a named barrier
// of their own; `slots` alternates between two buffers, so one barrier per sum is enough: a warp that writes a buffer
// again has passed the barrier in between, and so has everyone who read it.
template <int TW, int N>
__device__ __forceinline__ void ln_team_sum(float (&s)[N], float2 (*slots)[16], int& buf) {
#pragma unroll
    for (int o = (TW < 32 ? TW : 32) / 2; o; o >>= 1)
#pragma unroll
        for (int n = 0; n < N; ++n) s[n] += __shfl_xor_sync(0xffffffffu, s[n], o);
    if (TW > 32) {
        constexpr int W = TW / 32;
        const int warp = threadIdx.x >> 5, team = threadIdx.x / TW;
        if ((threadIdx.x & 31) == 0) slots[buf][warp] = make_float2(s[0], s[N - 1]);
        asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "n"(TW) : "memory");
        float2 v = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float2 o = slots[buf][team * W + w];
            v.x += o.x;
            v.y += o.y;
        }
        s[0] = v.x;
        if (N == 2) s[N - 1] = v.y;
        buf ^= 1;
    }
}

// The rows of a thread's team: r0, r0 + step, ...; `rows` of them.  `rounds` is the loop's length, the same for all threads that
// take part in a sum: teams narrower than a warp share it, so the last round may have no row for a team.
template <int TW>
struct LnRows {
    size_t r0, step;
    int rows, rounds;
    __device__ __forceinline__ LnRows(size_t M) {
        const int per_block = blockDim.x / TW;
        r0 = (size_t)blockIdx.x * per_block + threadIdx.x / TW;
        step = (size_t)gridDim.x * per_block;
        rows = r0 < M ? (int)((M - r0 - 1) / step + 1) : 0;
        const size_t w0 = TW >= 32 ? r0 : r0 - (threadIdx.x & 31) / TW;
        rounds = w0 < M ? (int)((M - w0 - 1) / step + 1) : 0;
    }
};

// A thread's channels: vector v holds c0 + v * TW * E .. + E - 1 where in(v); with PHASED, one more at cs where `single`.
template <int E, int TW, int MODE>
struct LnSpan {
    int lane, nvec, head, cs;
    bool single;
    template <typename T>
    __device__ __forceinline__ LnSpan(const T* row, int C) {
        lane = threadIdx.x % TW;
        head = MODE == LN_PHASED ? min(C, (int)(-(intptr_t)((uintptr_t)row / sizeof(T)) & (E - 1))) : 0;
        nvec = (C - head) / E;
        const int tail = head + nvec * E;
        cs = lane < E ? lane : tail + lane - E;
        single = MODE == LN_PHASED && (lane < E ? lane < head : cs < C);
    }
    __device__ __forceinline__ bool in(int v) const { return lane + v * TW < nvec; }
    __device__ __forceinline__ int channel(int v) const { return head + (lane + v * TW) * E; }
};

// A thread's vectors of the rows ahead, copied to shared memory by cp.async; each thread reads back only what it copied.
template <typename T, int E, int V, int TW, int MODE> struct LnRing {
    typedef LnSpan<E, TW, MODE> Span;
    static constexpr int B = E * (int)sizeof(T), BYTES = V * B;             // of a vector (16 or 8), of a row
    static __device__ __forceinline__ void request(uint32_t slot, int threads, const Span& at, const T* row, bool in) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (at.in(v)) cp_async<B>(slot + v * threads * B, row + at.channel(v), in);
    }
    // vectors past the row: never copied, zero throughout
    static __device__ __forceinline__ void zero(uint32_t slot, int threads, const Span& at) {
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (!at.in(v)) {
                if (B == 16) asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(slot + v * threads * B), "r"(0) : "memory");
                else asm volatile("st.shared.v2.b32 [%0], {%1, %1};" ::"r"(slot + v * threads * B), "r"(0) : "memory");
            }
    }
    static __device__ __forceinline__ void get(uint32_t slot, int threads, int v, float* f) {
        const uint32_t a = slot + v * threads * B;
        uint32_t u[4];
        if (B == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "r"(a) : "memory");
        else asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(u[0]), "=r"(u[1]) : "r"(a) : "memory");
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < E / 2; ++i) { f[2 * i] = bf16_lo(u[i]); f[2 * i + 1] = bf16_hi(u[i]); }
        } else {
#pragma unroll
            for (int i = 0; i < E; ++i) f[i] = __uint_as_float(u[i]);
        }
    }
};

// single elements (SINGLE), in registers, one row ahead
template <typename T, int V, int TW, int MODE>
struct LnAhead {
    T raw[V];
    __device__ __forceinline__ void request(const LnSpan<1, TW, MODE>& at, const T* row, bool in) {
#pragma unroll
        for (int v = 0; v < V; ++v) raw[v] = in && at.in(v) ? row[at.channel(v)] : T(0.f);
    }
};

template <typename TI, typename TO, int E, int V, int TW, int MODE>
__global__ void __launch_bounds__(TW > 256 ? TW : 256) ln_forward_kernel(const LnParams p) {
    constexpr bool RING = MODE != LN_SINGLE;
    constexpr int N = V * E + (MODE == LN_PHASED ? 2 : 0);          // a thread's channels; the single one and a zero last
    typedef LnRing<TI, E, V, TW, MODE> Ring;
    constexpr int S = ln_ring(Ring::BYTES);
    __shared__ float2 slots[2][16];
    extern __shared__ __align__(16) uint8_t ln_smem[];
    const uint32_t ring = ptx::smem_u32(ln_smem) + threadIdx.x * Ring::B;
    const int threads = blockDim.x, stage_bytes = Ring::BYTES * threads;
    int buf = 0;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const LnRows<TW> t(p.M);
    const TI* x = (const TI*)p.x + t.r0 * p.ldx;
    TO* y = (TO*)p.y + t.r0 * p.ldy;
    const size_t xstep = t.step * p.ldx, ystep = t.step * p.ldy;
    const LnSpan<E, TW, MODE> at(x, p.C);
    LnAhead<TI, RING ? 1 : V, TW, MODE> next;
    TI single = TI(0.f);
    const TI* xa = x;               // the next row to request
    if constexpr (MODE == LN_PHASED)
        if (at.single && t.rows > 0) single = x[at.cs];
    if constexpr (RING) {
#pragma unroll
        for (int k = 0; k < S; ++k) Ring::zero(ring + k * stage_bytes, threads, at);
#pragma unroll
        for (int k = 0; k < S - 1; ++k, xa += xstep) {
            if (k < t.rows) Ring::request(ring + k * stage_bytes, threads, at, xa, true);
            cp_async_commit();
        }
    } else {
        next.request(at, xa, t.rows > 0);
        xa += xstep;
    }
    alignas(8) float g[N], b[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool in = i < V * E ? at.in(i / E) : i == V * E && at.single;
        const int c = i < V * E ? at.channel(i / E) + i % E : at.cs;
        g[i] = p.gamma && in ? p.gamma[c] : 1.f;
        b[i] = p.beta && in ? p.beta[c] : 0.f;
    }
    float* mean_out = at.lane == 0 && p.mean ? p.mean + t.r0 : nullptr;
    float* rstd_out = at.lane == 0 && p.rstd ? p.rstd + t.r0 : nullptr;
    int cur = 0;
    for (int it = 0; it < t.rounds; ++it, x += xstep, y += ystep) {
        alignas(8) float f[N];
        if constexpr (RING) {
            int ahead = cur + S - 1;
            if (ahead >= S) ahead -= S;
            if (it + S - 1 < t.rows) Ring::request(ring + ahead * stage_bytes, threads, at, xa, true);
            xa += xstep;
            cp_async_commit();
            cp_async_wait<S - 1>();
#pragma unroll
            for (int v = 0; v < V; ++v) Ring::get(ring + cur * stage_bytes, threads, v, f + v * E);
            if (++cur == S) cur = 0;
            if constexpr (MODE == LN_PHASED) {
                f[V * E] = ln_value(single);
                f[V * E + 1] = 0.f;
                if (at.single && it + 1 < t.rows) single = x[xstep + at.cs];
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) f[v] = ln_value(next.raw[v]);
            next.request(at, xa, it + 1 < t.rows);
            xa += xstep;
        }
        float2 a = f2_at(f, 0);
#pragma unroll
        for (int i = 1; i < N / 2; ++i) a = f2_add(a, f2_at(f, i));
        float s[1] = {a.x + a.y};
        ln_team_sum<TW>(s, slots, buf);
        const float mean = s[0] * p.inv_c;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) f2_at(f, i) = f2_add(f2_at(f, i), f2(-mean));
        a = f2(0.f);
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (at.in(v)) {
                if constexpr (E > 1) {
#pragma unroll
                    for (int i = v * E / 2; i < (v + 1) * E / 2; ++i) a = f2_fma(f2_at(f, i), f2_at(f, i), a);
                } else {
                    a.x = fmaf(f[v], f[v], a.x);
                }
            }
        s[0] = a.x + a.y;
        if (MODE == LN_PHASED && at.single) s[0] = fmaf(f[V * E], f[V * E], s[0]);
        ln_team_sum<TW>(s, slots, buf);
        const float rstd = rsqrtf(fmaf(s[0], p.inv_c, p.eps));
        if (it < t.rows) {
#pragma unroll
            for (int i = 0; i < N / 2; ++i) f2_at(f, i) = f2_fma(f2_mul(f2_at(f, i), f2(rstd)), f2_at(g, i), f2_at(b, i));
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (at.in(v)) ln_store<E>(y + at.channel(v), f + v * E);
            if (MODE == LN_PHASED && at.single) ln_store1(y + at.cs, f[V * E]);
            if (mean_out) mean_out[it * t.step] = mean;
            if (rstd_out) rstd_out[it * t.step] = rstd;
        }
    }
}

// dx, and the block's sums of dy * xhat and of dy: every thread adds up its own channels over its rows in registers, the
// teams of a block are joined in shared memory in order, and the block writes one row of partial sums.  One block of 512
// threads per SM: the sums take 32 registers of a thread, and fewer, wider blocks leave fewer rows of partial sums to join
// (148 x 2 C floats).  As one cluster that joins its own sums, 49 x 1024 took 8.0 us instead of 8.2, but
// 196 x 512 and more rows took longer; the join stays a launch of its own.
template <typename TI, typename TO, int E, int V, int TW, int MODE>
__global__ void __launch_bounds__(LN_BWD_THREADS, 1) ln_backward_kernel(const LnParams p) {
    constexpr bool RING = MODE != LN_SINGLE;
    constexpr int N = V * E + (MODE == LN_PHASED ? 2 : 0);
    typedef LnRing<TI, E, V, TW, MODE> RX;
    typedef LnRing<TO, E, V, TW, MODE> RD;
    constexpr int S = ln_ring(RX::BYTES + RD::BYTES), T = LN_BWD_THREADS;
    constexpr int STAGE = (RX::BYTES + RD::BYTES + 8) * T;         // and the row's mean and rstd
    __shared__ float2 slots[2][16];
    extern __shared__ __align__(16) uint8_t ln_smem[];          // the ring; afterwards [teams][2][C] sums
    const uint32_t smem = ptx::smem_u32(ln_smem);
    const uint32_t ringx = smem + threadIdx.x * RX::B, ringd = smem + RX::BYTES * T + threadIdx.x * RD::B;
    // mean and rstd are copied by one thread of the team (of each of its warps): the others read them after __syncwarp
    const int lead = threadIdx.x & ~((TW < 32 ? TW : 32) - 1);
    const uint32_t rings = smem + (RX::BYTES + RD::BYTES) * T + lead * 8;
    int buf = 0;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const LnRows<TW> t(p.M);
    const TI* x = (const TI*)p.x + t.r0 * p.ldx;
    const TO* dy = (const TO*)p.dy + t.r0 * p.ldy;
    TI* dx = (TI*)p.dx + t.r0 * p.lddx;
    const size_t xstep = t.step * p.ldx, dstep = t.step * p.ldy, ostep = t.step * p.lddx;
    const LnSpan<E, TW, MODE> at(x, p.C);
    LnAhead<TI, RING ? 1 : V, TW, MODE> nx;
    LnAhead<TO, RING ? 1 : V, TW, MODE> nd;
    TI sx = TI(0.f);
    TO sd = TO(0.f);
    float nmean = 0.f, nrstd = 0.f;
    const TI* xa = x;
    const TO* da = dy;
    const float *ma = p.mean_in + t.r0, *ra = p.rstd_in + t.r0;
    if constexpr (MODE == LN_PHASED)
        if (at.single && t.rows > 0) { sx = x[at.cs]; sd = dy[at.cs]; }
    auto request = [&](int stage, bool in) {
        // past the last row: zeros, so that a team without a row in the warp's last round adds nothing
        RX::request(ringx + stage * STAGE, T, at, in ? xa : (const TI*)p.x, in);
        RD::request(ringd + stage * STAGE, T, at, in ? da : (const TO*)p.dy, in);
        if ((int)threadIdx.x == lead) {
            cp_async<4>(rings + stage * STAGE, in ? ma : p.mean_in, in);
            cp_async<4>(rings + stage * STAGE + 4, in ? ra : p.rstd_in, in);
        }
        cp_async_commit();
        xa += xstep;
        da += dstep;
        ma += t.step;
        ra += t.step;
    };
    if constexpr (RING) {
#pragma unroll
        for (int k = 0; k < S; ++k) {
            RX::zero(ringx + k * STAGE, T, at);
            RD::zero(ringd + k * STAGE, T, at);
        }
#pragma unroll
        for (int k = 0; k < S - 1; ++k) request(k, k < t.rows);
    } else {
        nx.request(at, x, t.rows > 0);
        nd.request(at, dy, t.rows > 0);
        if (t.rows > 0) { nmean = *ma; nrstd = *ra; }
    }
    alignas(8) float g[N], sg[N], sb[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool in = i < V * E ? at.in(i / E) : i == V * E && at.single;
        g[i] = p.gamma && in ? p.gamma[i < V * E ? at.channel(i / E) + i % E : at.cs] : 1.f;
        sg[i] = sb[i] = 0.f;
    }
    int cur = 0;
    for (int it = 0; it < t.rounds; ++it, x += xstep, dy += dstep, dx += ostep) {
        alignas(8) float h[N], d[N];
        float mean = nmean, rstd = nrstd;
        const bool more = it + 1 < t.rows;
        if constexpr (RING) {
            int ahead = cur + S - 1;
            if (ahead >= S) ahead -= S;
            request(ahead, it + S - 1 < t.rows);
            cp_async_wait<S - 1>();
            __syncwarp();
#pragma unroll
            for (int v = 0; v < V; ++v) {
                RX::get(ringx + cur * STAGE, T, v, h + v * E);
                RD::get(ringd + cur * STAGE, T, v, d + v * E);
            }
            asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(mean), "=f"(rstd) : "r"(rings + cur * STAGE) : "memory");
            if (++cur == S) cur = 0;
            if constexpr (MODE == LN_PHASED) {
                h[V * E] = ln_value(sx);
                d[V * E] = ln_value(sd);
                h[V * E + 1] = d[V * E + 1] = 0.f;
                sd = TO(0.f);
                if (at.single && more) { sx = x[xstep + at.cs]; sd = dy[dstep + at.cs]; }
            }
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                h[v] = ln_value(nx.raw[v]);
                d[v] = ln_value(nd.raw[v]);
            }
            nx.request(at, x + xstep, more);
            nd.request(at, dy + dstep, more);
            nmean = more ? ma[(it + 1) * t.step] : 0.f;
            nrstd = more ? ra[(it + 1) * t.step] : 0.f;
        }
        // Channels past the row have x = dy = 0, and so no part in any sum, unless mean * rstd passes float32's range: then x = mean there.
        // (46000 x 1101 98 -> 100 us by this test, 122 by a select for each vector, 125 by leaving the empty vectors out; 154000 x 333 77 -> 77, 76, 100.)
        if (!(fabsf(mean * rstd) < INFINITY)) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i < V * E ? !at.in(i / E) : i > V * E || !at.single) h[i] = mean;
        }
        float2 s1 = f2(0.f), s2 = s1;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            // x - mean first: x rstd - mean rstd would lose what a row far from zero has left
            const float2 hv = f2_mul(f2_add(f2_at(h, i), f2(-mean)), f2(rstd)), dv = f2_at(d, i);
            f2_at(sg, i) = f2_fma(dv, hv, f2_at(sg, i));
            f2_at(sb, i) = f2_add(f2_at(sb, i), dv);
            const float2 tv = f2_mul(dv, f2_at(g, i));
            s1 = f2_add(s1, tv);
            s2 = f2_fma(tv, hv, s2);
            f2_at(h, i) = hv;
            f2_at(d, i) = tv;
        }
        float s[2] = {s1.x + s1.y, s2.x + s2.y};
        ln_team_sum<TW>(s, slots, buf);
        if (it < t.rows) {
            const float2 m1 = f2(-s[0] * p.inv_c), m2 = f2(-s[1] * p.inv_c);
#pragma unroll
            for (int i = 0; i < N / 2; ++i) f2_at(d, i) = f2_mul(f2(rstd), f2_add(f2_at(d, i), f2_fma(f2_at(h, i), m2, m1)));
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (at.in(v)) ln_store<E>(dx + at.channel(v), d + v * E);
            if (MODE == LN_PHASED && at.single) ln_store1(dx + at.cs, d[V * E]);
        }
    }
    if (!p.partials) return;
    if constexpr (RING) {
        cp_async_wait<0>();
        __syncthreads();                        // every thread is done with the ring
    }
    float* red = reinterpret_cast<float*>(ln_smem);
    float* mine = red + (size_t)(threadIdx.x / TW) * 2 * p.C;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool in = i < V * E ? at.in(i / E) : i == V * E && at.single;
        const int c = i < V * E ? at.channel(i / E) + i % E : at.cs;
        if (in) {
            mine[c] = sg[i];
            mine[p.C + c] = sb[i];
        }
    }
    __syncthreads();
    float* out = p.partials + (size_t)blockIdx.x * 2 * p.C;
    for (int i = threadIdx.x; i < 2 * p.C; i += T) {
        float s = 0.f;
#pragma unroll 4
        for (int k = 0; k < T / TW; ++k) s += red[(size_t)k * 2 * p.C + i];
        out[i] = s;
    }
}

// Rows too long for a team's registers: a block walks its row from memory (the second and third time from L2), and the
// weight gradients of its rows are added up in its own row of partial sums, each channel always by the same thread.
template <typename TI, typename TO>
__global__ void __launch_bounds__(512) ln_forward_long_kernel(const LnParams p) {
    __shared__ float2 slots[2][16];
    const unsigned C = p.C;                     // positions past C, and the backward pass' second half of sums, pass 31 bits
    int buf = 0;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    for (size_t r = blockIdx.x; r < p.M; r += gridDim.x) {
        float s[1] = {0.f};
        for (unsigned c = threadIdx.x; c < C; c += 512) s[0] += ln_value(((const TI*)p.x)[r * p.ldx + c]);
        ln_team_sum<512>(s, slots, buf);
        const float mean = s[0] * p.inv_c;
        s[0] = 0.f;
        for (unsigned c = threadIdx.x; c < C; c += 512) {
            const float d = ln_value(((const TI*)p.x)[r * p.ldx + c]) - mean;
            s[0] = fmaf(d, d, s[0]);
        }
        ln_team_sum<512>(s, slots, buf);
        const float rstd = rsqrtf(fmaf(s[0], p.inv_c, p.eps));
        for (unsigned c = threadIdx.x; c < C; c += 512) {
            const float v = fmaf((ln_value(((const TI*)p.x)[r * p.ldx + c]) - mean) * rstd, p.gamma ? p.gamma[c] : 1.f, p.beta ? p.beta[c] : 0.f);
            ln_store1((TO*)p.y + r * p.ldy + c, v);
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
    }
}

template <typename TI, typename TO>
__global__ void __launch_bounds__(512) ln_backward_long_kernel(const LnParams p) {
    __shared__ float2 slots[2][16];
    const unsigned C = p.C;                     // positions past C, and the backward pass' second half of sums, pass 31 bits
    int buf = 0;
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    float* sg = p.partials ? p.partials + (size_t)blockIdx.x * 2 * C : nullptr;
    float* sb = sg ? sg + C : nullptr;
    if (sg)
        for (unsigned c = threadIdx.x; c < C; c += 512) sg[c] = sb[c] = 0.f;
    for (size_t r = blockIdx.x; r < p.M; r += gridDim.x) {
        const float mean = p.mean_in[r], rstd = p.rstd_in[r];
        float s[2] = {0.f, 0.f};
        for (unsigned c = threadIdx.x; c < C; c += 512) {
            const float d = ln_value(((const TO*)p.dy)[r * p.ldy + c]), h = (ln_value(((const TI*)p.x)[r * p.ldx + c]) - mean) * rstd;
            const float t = d * (p.gamma ? p.gamma[c] : 1.f);
            s[0] += t;
            s[1] = fmaf(t, h, s[1]);
            if (sg) {
                sg[c] = fmaf(d, h, sg[c]);
                sb[c] += d;
            }
        }
        ln_team_sum<512>(s, slots, buf);
        s[0] *= p.inv_c;
        s[1] *= p.inv_c;
        for (unsigned c = threadIdx.x; c < C; c += 512) {
            const float t = ln_value(((const TO*)p.dy)[r * p.ldy + c]) * (p.gamma ? p.gamma[c] : 1.f), h = (ln_value(((const TI*)p.x)[r * p.ldx + c]) - mean) * rstd;
            const float v = rstd * (t - fmaf(h, s[1], s[0]));
            ln_store1((TI*)p.dx + r * p.lddx + c, v);
        }
    }
}

// dgamma and dbeta: the blocks' partial sums in a fixed order, 16 ranges of them side by side
__global__ void __launch_bounds__(512) ln_join_kernel(const LnParams p) {
    __shared__ float red[16][32];
    ptx::grid_dependency_wait();
    ptx::grid_launch_dependents();
    const size_t C = p.C, i = (size_t)blockIdx.x * 32 + (threadIdx.x & 31);
    const int q = threadIdx.x >> 5;
    float s = 0.f;
    if (i < 2 * C) {
#pragma unroll 10
        for (int k = q; k < p.n_part; k += 16) s += p.partials[k * 2 * C + i];
    }
    red[q][threadIdx.x & 31] = s;
    __syncthreads();
    if (q == 0 && i < 2 * C) {
#pragma unroll
        for (int k = 1; k < 16; ++k) s += red[k][threadIdx.x];
        float* out = i < C ? p.dgamma : p.dbeta;
        if (out) out[i < C ? i : i - C] = s;
    }
}

// ------------------------------------------------------------------------------------------------ host side
typedef void (*LnKernel)(const LnParams);
struct LnChoice {
    LnKernel kernel;
    int tw, mode, ring;             // threads per row (0: the long-row kernel), LN_*, ring bytes per thread
};

template <bool BWD, typename TI, typename TO, int E, int V, int TW, int MODE>
static LnChoice ln_pick() {
    constexpr int row = LnRing<TI, E, V, TW, MODE>::BYTES + (BWD ? LnRing<TO, E, V, TW, MODE>::BYTES : 0);
    constexpr int ring = MODE != LN_SINGLE ? (row + (BWD ? 8 : 0)) * ln_ring(row) : 0;
    if constexpr (BWD) return {ln_backward_kernel<TI, TO, E, V, TW, MODE>, TW, MODE, ring};
    else return {ln_forward_kernel<TI, TO, E, V, TW, MODE>, TW, MODE, ring};
}

// The narrowest team whose registers hold the row, 16 channels a thread: fewer threads per row mean fewer steps in its
// sums and fewer registers spent on half-empty vectors.  PHASED: at least 2 E threads, one for each channel outside the vectors.
// Forward, rows a little too long for a team get 24 channels a thread instead of a team of twice the size that is mostly empty (bfloat16,
// 154000 rows of 333, phased: 58 -> 42 us; 46000 of 1104: 54 -> 42 us; 24000 of 2100: 84 -> 46 us; 1536, three quarters full: 41 -> 37 us;
// with float32 vectors of 4, 333: 64 -> 55 us, but 1400: 50 -> 53 us, so only up to a third more).  The backward pass would not fit its registers.
template <bool BWD, typename TI, typename TO, int MODE>
static LnChoice ln_pick_vec(int C) {
    constexpr int E = sizeof(TI) + sizeof(TO) == 4 ? 8 : 4, V = 16 / E, W = MODE == LN_PHASED ? 2 * E : 8;
    if (C <= 8 * W) return ln_pick<BWD, TI, TO, E, V / 2, W, MODE>();
    if (C <= 128) return ln_pick<BWD, TI, TO, E, V, W, MODE>();
    if (C <= 256) return ln_pick<BWD, TI, TO, E, V, 16, MODE>();
    if constexpr (!BWD) {
        auto more = [&](int full) { return C > full && C <= full + (E == 8 ? full / 2 : full / 3); };
        if (more(256)) return ln_pick<BWD, TI, TO, E, 3 * V / 2, 16, MODE>();
        if (more(512)) return ln_pick<BWD, TI, TO, E, 3 * V / 2, 32, MODE>();
        if (more(1024)) return ln_pick<BWD, TI, TO, E, 3 * V / 2, 64, MODE>();
        if (more(2048)) return ln_pick<BWD, TI, TO, E, 3 * V / 2, 128, MODE>();
        if (more(4096)) return ln_pick<BWD, TI, TO, E, 3 * V / 2, 256, MODE>();
    }
    if (C <= 512) return ln_pick<BWD, TI, TO, E, V, 32, MODE>();
    if (C <= 1024) return ln_pick<BWD, TI, TO, E, V, 64, MODE>();
    if (C <= 2048) return ln_pick<BWD, TI, TO, E, V, 128, MODE>();
    if (C <= 4096) return ln_pick<BWD, TI, TO, E, V, 256, MODE>();
    if constexpr (BWD) return ln_pick<BWD, TI, TO, E, V, 512, MODE>();
    else return ln_pick<BWD, TI, TO, E, 2 * V, 256, MODE>();
}
template <bool BWD, typename TI, typename TO>
static LnChoice ln_choose(int C, int mode) {
    if (mode == LN_ALIGNED && C <= 8192) return ln_pick_vec<BWD, TI, TO, LN_ALIGNED>(C);
    if (mode == LN_PHASED && C <= 8192) return ln_pick_vec<BWD, TI, TO, LN_PHASED>(C);
    if (C <= 256) return ln_pick<BWD, TI, TO, 1, 8, 32, LN_SINGLE>();
    if (C <= 512) return ln_pick<BWD, TI, TO, 1, 8, 64, LN_SINGLE>();
    if (C <= 1024) return ln_pick<BWD, TI, TO, 1, 8, 128, LN_SINGLE>();
    if (C <= 4096) return ln_pick<BWD, TI, TO, 1, 8, 512, LN_SINGLE>();
    if constexpr (BWD) return {ln_backward_long_kernel<TI, TO>, 0, LN_SINGLE, 0};
    else return {ln_forward_long_kernel<TI, TO>, 0, LN_SINGLE, 0};
}
template <bool BWD>
static LnChoice ln_choose(int C, int mode, unsigned flags) {
    const bool xf = flags & DR_LN_X_F32, yf = flags & DR_LN_Y_F32;
    if (xf) return yf ? ln_choose<BWD, float, float>(C, mode) : ln_choose<BWD, float, __nv_bfloat16>(C, mode);
    return yf ? ln_choose<BWD, __nv_bfloat16, float>(C, mode) : ln_choose<BWD, __nv_bfloat16, __nv_bfloat16>(C, mode);
}

// Rows of partial sums that the workspace is sized for: one for each block of the backward pass, and that has one block per SM
// (its registers fill it), or fewer where the rows do not give every team one.
static int ln_parts(size_t M) { return (int)(M < 1 ? 1 : M < (size_t)num_sms() ? M : (size_t)num_sms()); }
static bool ln_aligned(const void* p, bool f32) { return ((uintptr_t)p & (f32 ? 3u : 1u)) == 0; }

// the mode of a call whose tensors have these addresses and row strides (in elements of 4 or 2 bytes)
struct LnRowsAt { const void* p; int ld; bool f32; };
static int ln_mode(int C, std::initializer_list<LnRowsAt> ts) {
    unsigned mask = 7;                          // elements of a vector, less one
    for (const LnRowsAt& t : ts)
        if (t.f32) mask = 3;
    bool aligned = (C & mask) == 0, phased = true;
    const LnRowsAt& a = *ts.begin();
    const uintptr_t first = (uintptr_t)a.p / (a.f32 ? 4 : 2);
    for (const LnRowsAt& t : ts) {
        const uintptr_t at = (uintptr_t)t.p / (t.f32 ? 4 : 2);
        aligned = aligned && (at & mask) == 0 && (t.ld & mask) == 0;
        phased = phased && ((at - first) & mask) == 0 && ((t.ld - a.ld) & mask) == 0;
    }
    return aligned ? LN_ALIGNED : phased ? LN_PHASED : LN_SINGLE;
}
// blocks of a launch: at most `cap`, no more than the rows need; PHASED: the number of teams a multiple of 8
static size_t ln_blocks(const LnChoice& c, int threads, size_t rows, size_t cap) {
    const size_t per = c.tw ? (size_t)(threads / c.tw) : 1, need = (rows + per - 1) / per;
    if (need <= cap) return need;               // one round: a team has one row
    if (c.mode == LN_PHASED && per < 8) cap -= cap % (8 / per);
    return cap;
}

}  // namespace dr

using namespace dr;

// Blocks of `threads` threads and `smem` bytes an SM holds.  The opt-in to more shared memory and the answer belong to the
// current device: asked once per kernel, size and device.
static int ln_ask_blocks_per_sm(LnKernel k, int threads, size_t smem) {
    int n = 0;
    // always to the most any call of any of the kernels asks for, so that a later call does not lower it
    if (smem > LN_SMEM_MAX || cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)LN_SMEM_MAX) != cudaSuccess ||
        cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, k, threads, smem) != cudaSuccess || n < 1) {
        (void)cudaGetLastError();
        return 0;
    }
    return n;
}
static int ln_blocks_per_sm(LnKernel k, int threads, size_t smem) {
    static std::mutex mu;
    static std::map<std::tuple<LnKernel, size_t, int>, int> known;
    try {
        std::lock_guard<std::mutex> lock(mu);
        const auto key = std::make_tuple(k, smem, PerDeviceFlag::dev());
        const auto it = known.find(key);
        if (it != known.end()) return it->second;
        const int n = ln_ask_blocks_per_sm(k, threads, smem);
        return n ? known[key] = n : 0;
    } catch (...) {             // no memory for the table: nothing may leave a C entry
        return ln_ask_blocks_per_sm(k, threads, smem);
    }
}

// Launched with programmatic serialization: the block set-up overlaps the tail of the kernel in front, which every kernel
// here waits for before its first access to memory.
static int ln_launch(LnKernel k, size_t blocks, int threads, size_t smem, const LnParams& p, void* stream) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.gridDim = dim3((unsigned)blocks); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = (cudaStream_t)stream;
    cfg.attrs = attr; cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, k, p) != cudaSuccess) { (void)cudaGetLastError(); return DR_ERR_CUDA; }
    count_launch();
    return launch_status();
}

extern "C" int dr_layernorm(size_t npix, int C, const void* x, int ldx, const float* gamma, const float* beta, float eps, void* y, int ldy,
                            float* mean, float* rstd, unsigned flags, void* stream) {
    if (!x || !y || C <= 0 || !(eps >= 0.f) || (flags & ~(unsigned)(DR_LN_X_F32 | DR_LN_Y_F32))) return DR_ERR_INVALID_ARG;
    if (ldx == 0) ldx = C;
    if (ldy == 0) ldy = C;
    if (ldx < C || ldy < C) return DR_ERR_INVALID_ARG;
    if (!ln_aligned(x, flags & DR_LN_X_F32) || !ln_aligned(y, flags & DR_LN_Y_F32) || !ln_aligned(gamma, true) || !ln_aligned(beta, true) ||
        !ln_aligned(mean, true) || !ln_aligned(rstd, true)) return DR_ERR_ALIGNMENT;
    if (npix == 0) return DR_OK;
    LnParams p = {};
    p.M = npix; p.C = C; p.x = x; p.ldx = ldx; p.gamma = gamma; p.beta = beta; p.eps = eps; p.y = y; p.ldy = ldy; p.mean = mean; p.rstd = rstd;
    p.inv_c = 1.f / (float)C;
    const LnChoice c = ln_choose<false>(C, ln_mode(C, {{x, ldx, (flags & DR_LN_X_F32) != 0}, {y, ldy, (flags & DR_LN_Y_F32) != 0}}), flags);
    const int threads = c.tw == 0 ? 512 : c.tw > 256 ? c.tw : 256;
    const size_t smem = (size_t)c.ring * threads;
    const int per_sm = ln_blocks_per_sm(c.kernel, threads, smem);
    if (per_sm < 1) return DR_ERR_CUDA;
    return ln_launch(c.kernel, ln_blocks(c, threads, npix, (size_t)num_sms() * per_sm), threads, smem, p, stream);
}

extern "C" int dr_layernorm_bwd_workspace_bytes(size_t npix, int C, size_t* bytes) {
    if (!bytes || C <= 0) return DR_ERR_INVALID_ARG;
    *bytes = ((size_t)ln_parts(npix) * 2 * C * sizeof(float) + 255) / 256 * 256;
    return DR_OK;
}

extern "C" int dr_layernorm_bwd(size_t npix, int C, const void* dy, int lddy, const void* x, int ldx, const float* gamma, const float* mean,
                                const float* rstd, void* dx, int lddx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes,
                                unsigned flags, void* stream) {
    if (!x || !dy || !dx || !mean || !rstd || C <= 0 || (flags & ~(unsigned)(DR_LN_X_F32 | DR_LN_Y_F32))) return DR_ERR_INVALID_ARG;
    if (lddy == 0) lddy = C;
    if (ldx == 0) ldx = C;
    if (lddx == 0) lddx = C;
    if (lddy < C || ldx < C || lddx < C) return DR_ERR_INVALID_ARG;
    const bool sums = dgamma || dbeta;
    if (sums && !workspace) return DR_ERR_INVALID_ARG;
    const bool xf = flags & DR_LN_X_F32, yf = flags & DR_LN_Y_F32;
    if (!ln_aligned(x, xf) || !ln_aligned(dx, xf) || !ln_aligned(dy, yf) || !ln_aligned(gamma, true) || !ln_aligned(mean, true) ||
        !ln_aligned(rstd, true) || !ln_aligned(dgamma, true) || !ln_aligned(dbeta, true) || (sums && ((uintptr_t)workspace & 255))) return DR_ERR_ALIGNMENT;
    size_t need = 0;
    dr_layernorm_bwd_workspace_bytes(npix, C, &need);
    if (sums && workspace_bytes < need) return DR_ERR_WORKSPACE;
    if (sums && dgamma == dbeta) return DR_ERR_INVALID_ARG;         // two writers of one buffer
    cudaStream_t s = (cudaStream_t)stream;
    if (npix == 0) {            // an empty sum
        if (dgamma && cudaMemsetAsync(dgamma, 0, (size_t)C * sizeof(float), s) != cudaSuccess) return DR_ERR_CUDA;
        if (dbeta && cudaMemsetAsync(dbeta, 0, (size_t)C * sizeof(float), s) != cudaSuccess) return DR_ERR_CUDA;
        return DR_OK;
    }
    LnParams p = {};
    p.M = npix; p.C = C; p.dy = dy; p.ldy = lddy; p.x = x; p.ldx = ldx; p.gamma = gamma; p.mean_in = mean; p.rstd_in = rstd; p.dx = dx; p.lddx = lddx;
    p.partials = sums ? (float*)workspace : nullptr; p.dgamma = dgamma; p.dbeta = dbeta; p.inv_c = 1.f / (float)C;
    const LnChoice c = ln_choose<true>(C, ln_mode(C, {{x, ldx, xf}, {dy, lddy, yf}, {dx, lddx, xf}}), flags);
    p.n_part = (int)ln_blocks(c, LN_BWD_THREADS, npix, (size_t)num_sms());
    const size_t join = c.tw && sums ? (size_t)(LN_BWD_THREADS / c.tw) * 2 * C * sizeof(float) : 0;
    const size_t smem = std::max((size_t)c.ring * LN_BWD_THREADS, join);
    if (ln_blocks_per_sm(c.kernel, LN_BWD_THREADS, smem) < 1) return DR_ERR_CUDA;
    const int st = ln_launch(c.kernel, (size_t)p.n_part, LN_BWD_THREADS, smem, p, stream);
    if (st != DR_OK || !sums) return st;
    return ln_launch(ln_join_kernel, (2 * (size_t)C + 31) / 32, 512, 0, p, stream);
}
