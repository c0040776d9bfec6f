// What the kernels of the orthogonalised update share: the input, the optimiser's element-wise part, float16 pairs.
#pragma once
#include <cuda_fp16.h>

#include "conv_common.cuh"
#include "umma_ptx.cuh"

namespace dr {
using namespace ptx;

// X is stored times this: entries from 1.5e-8 on are in float16's normal range, their low halves from 6e-5 on; smaller ones have fewer bits, and an
// absolute error of at most 7e-12.
constexpr float NS_SCALE = 4096.f;

// Shared memory every CTA asks for, whether it needs it or not.  CTAs here wait for one another at cluster and grid barriers, so none of them may
// have to wait for tensor memory that another CTA on its SM holds (and that one perhaps for a CTA of its own).  Today's registers (384
// threads of 168, 512 of 128) leave no room for another CTA anyway; with this, no kernel that uses tensor memory fits beside one of these
// whatever registers a compiler gives.  All 227 KB cost cache: 4096 x 9216 2.34 ms against 2.07, 192 x 576 105
// against 102 us.
constexpr int NS_SMEM_ALL = 193 * 1024;

struct NsInput {
    int rows, cols, tall;
    const void* g;              // gradient (bfloat16 or float32), or the optimiser's float32 gradient
    int g_f32;
    float *v, *w;               // optimiser state, nullptr for the product alone
    float momentum;
    int nesterov;
    float eps;
    float lr_scale, keep;       // w <- keep w - lr_scale O
    __nv_bfloat16* out;         // O, or the bfloat16 copy of w (may be nullptr then)
    int vec;                    // rows of a multiple of 8 elements at 16-byte aligned addresses: 16-byte accesses
};

__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile("{\n.reg .pred P;\nelect.sync _|P, 0xffffffff;\nselp.u32 %0, 1, 0, P;\n}" : "=r"(e));
    return e != 0;
}

__device__ __forceinline__ int cluster_ctas() {
    uint32_t n;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(n));
    return (int)n;
}
// A launch that lost its cluster size (a profiler that replays a cooperative launch, say) must not reach an instruction for clusters or CTA
// pairs, nor a neighbour's shared memory: the kernels ask this first, and return.
__device__ __forceinline__ bool cluster_lost(int ctas, int* status) {
    if (cluster_ctas() == ctas) return false;
    if (threadIdx.x == 0) report_timeout(status, 77, ctas);
    return true;
}

struct __align__(32) Half16 { uint32_t u[8]; };
struct __align__(32) Float8 { float f[8]; };
__device__ __forceinline__ Half16 ld16h(const __half* p) {
    Half16 v;
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=r"(v.u[0]), "=r"(v.u[1]), "=r"(v.u[2]), "=r"(v.u[3]), "=r"(v.u[4]), "=r"(v.u[5]), "=r"(v.u[6]), "=r"(v.u[7]) : "l"(p) : "memory");
    return v;
}
__device__ __forceinline__ void st16h(__half* p, const Half16& v) {
    asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"r"(v.u[0]), "r"(v.u[1]), "r"(v.u[2]), "r"(v.u[3]), "r"(v.u[4]), "r"(v.u[5]), "r"(v.u[6]), "r"(v.u[7]), "l"(p) : "memory");
}
__device__ __forceinline__ void ld8f(const float* p, float* f) {
    asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];" : "=f"(f[0]), "=f"(f[1]), "=f"(f[2]), "=f"(f[3]), "=f"(f[4]), "=f"(f[5]), "=f"(f[6]), "=f"(f[7]) : "l"(p) : "memory");
}
__device__ __forceinline__ void st8f(float* p, const float* f) {
    asm volatile("st.global.v8.f32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::"f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]), "l"(p) : "memory");
}
__device__ __forceinline__ float2 half2_at(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// v as float16 h and what that leaves out as float16 l
template <int CN>
__device__ __forceinline__ void ns_split(const float* v, uint32_t* h, uint32_t* l) {
#pragma unroll
    for (int c = 0; c < CN; c += 2) {
        h[c / 2] = pack_half(v[c], v[c + 1]);
        const float2 f = half2_at(h[c / 2]);
        l[c / 2] = pack_half(v[c] - f.x, v[c + 1] - f.y);
    }
}

// CN consecutive values of U: from the gradient, or from the updated momentum and, with Nesterov, the gradient
template <int CN, typename T> __device__ __forceinline__ void ns_read(const T* p, float* f);
template <> __device__ __forceinline__ void ns_read<1, float>(const float* p, float* f) { f[0] = *p; }
template <> __device__ __forceinline__ void ns_read<1, __nv_bfloat16>(const __nv_bfloat16* p, float* f) { f[0] = __bfloat162float(*p); }
template <> __device__ __forceinline__ void ns_read<8, float>(const float* p, float* f) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
template <> __device__ __forceinline__ void ns_read<8, __nv_bfloat16>(const __nv_bfloat16* p, float* f) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    f[0] = bf16_lo(a.x); f[1] = bf16_hi(a.x); f[2] = bf16_lo(a.y); f[3] = bf16_hi(a.y);
    f[4] = bf16_lo(a.z); f[5] = bf16_hi(a.z); f[6] = bf16_lo(a.w); f[7] = bf16_hi(a.w);
}
template <int CN> __device__ __forceinline__ void ns_write(float* p, const float* f) {
    if (CN == 8) {
        reinterpret_cast<float4*>(p)[0] = make_float4(f[0], f[1 % CN], f[2 % CN], f[3 % CN]);
        reinterpret_cast<float4*>(p)[1] = make_float4(f[4 % CN], f[5 % CN], f[6 % CN], f[7 % CN]);
    } else {
        *p = f[0];
    }
}
template <int CN> __device__ __forceinline__ void ns_write(__nv_bfloat16* p, const float* f) {
    if (CN == 8) *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16(f[0], f[1 % CN]), pack_bf16(f[2 % CN], f[3 % CN]), pack_bf16(f[4 % CN], f[5 % CN]), pack_bf16(f[6 % CN], f[7 % CN]));
    else *p = __float2bfloat16_rn(f[0]);
}
template <int CN>
__device__ __forceinline__ void ns_value(const NsInput& in, size_t i, float* u) {
    if (in.v) {
        ns_read<CN>(in.v + i, u);
        if (in.nesterov) {
            float g[CN];
            ns_read<CN>((const float*)in.g + i, g);
#pragma unroll
            for (int c = 0; c < CN; ++c) u[c] = fmaf(in.momentum, u[c], g[c]);
        }
    } else if (in.g_f32) {
        ns_read<CN>((const float*)in.g + i, u);
    } else {
        ns_read<CN>((const __nv_bfloat16*)in.g + i, u);
    }
}

// v <- momentum v + g and this thread's part of the sum of squares of U (in float64: no size of U overflows or vanishes)
template <int CN>
__device__ __forceinline__ double ns_momentum_part(const NsInput& in, size_t base, size_t count, size_t first, size_t stride) {
    double s = 0.;
    for (size_t i = first; i < count; i += stride) {
        float u[CN], g[CN];
        if (in.v) {
            ns_read<CN>(in.v + base + i * CN, u);
            ns_read<CN>((const float*)in.g + base + i * CN, g);
#pragma unroll
            for (int c = 0; c < CN; ++c) u[c] = fmaf(in.momentum, u[c], g[c]);
            ns_write<CN>(in.v + base + i * CN, u);
            if (in.nesterov) {
#pragma unroll
                for (int c = 0; c < CN; ++c) u[c] = fmaf(in.momentum, u[c], g[c]);
            }
        } else {
            ns_value<CN>(in, base + i * CN, u);
        }
#pragma unroll
        for (int c = 0; c < CN; ++c) s = fma((double)u[c], (double)u[c], s);
    }
    return s;
}
__device__ __forceinline__ double ns_momentum(const NsInput& in, size_t base, size_t per, size_t first, size_t stride) {
    return in.vec ? ns_momentum_part<8>(in, base, per / 8, first, stride) : ns_momentum_part<1>(in, base, per, first, stride);
}

__device__ __forceinline__ double ns_warp_sum(double s) {
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// X_0 = U / (|U|_F + eps), times NS_SCALE: u * first * second.  The quotient alone leaves float32's normal range where the norm is below 1.2e-35 or
// above 3.4e41; a power of two in front (exact, but for entries 2^-110 times the norm) keeps both factors inside it for every size of U.
struct NsFactor { float first, second; };
__device__ __forceinline__ NsFactor ns_factor(double squares, float eps) {
    const double d = sqrt(squares) + (double)eps;
    const double first = d < 0x1p-64 ? 0x1p100 : d > 0x1p64 ? 0x1p-80 : 1.;
    return {(float)first, (float)((double)NS_SCALE / (d * first))};
}

// 8 (or 1) values of the result: O, or the update of w
template <int CN>
__device__ __forceinline__ void ns_put_o(const NsInput& in, size_t at, float* o) {
    if (in.w) {
        float w[CN];
        ns_read<CN>(in.w + at, w);
#pragma unroll
        for (int c = 0; c < CN; ++c) o[c] = fmaf(-in.lr_scale, o[c], in.keep * w[c]);
        ns_write<CN>(in.w + at, o);
    }
    if (in.out) ns_write<CN>(in.out + at, o);
}
// The kernel for matrices of at most 128 rows that a cluster holds in shared memory (muon_small.cu); 0 CTAs: not for this shape.
struct NsSmallPlan { int ctas, groups, chunks, terms; size_t part, sums, diag, bytes; };
NsSmallPlan ns_small_plan(int batch, int rows, int cols);
int ns_small_lost_cluster(cudaStream_t stream);         // self-test, see dr_selftest_lost_cluster
int ns_small_run(const NsSmallPlan& plan, int batch, const NsInput& in, int steps, const float* coef, void* workspace, cudaStream_t stream);

}  // namespace dr
