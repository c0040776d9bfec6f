// The dropout's counter-based generator, shared by the kernels that draw a mask or draw it again.
//
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", 2011) under the key `seed`.  Elements e of a
// row-major [rows][channels] tensor are numbered by e = row * channels + channel whatever the tensor's strides; counter (e / 8, offset)
// gives four words, and element e takes 16 bits of them: word (e mod 8) / 2, the low half first.  It is dropped where these are below
// thr = round(p * 65536).  Sixteen bits an element instead of 32 halve the generator's arithmetic, which would otherwise cost as much time as the
// memory (a call is about 60 issue slots, 16-bit tensors leave about 20 an element); the kept ones are scaled by 65536 / (65536 - thr),
// so that the expectation is exact for the probability that is drawn.
#pragma once
#include <math.h>
#include <stdint.h>

namespace dr {

struct DropKey {
    uint32_t k0, k1;                    // seed
    unsigned long long offset;
    const unsigned long long* step;     // nullptr, or a counter in device memory that is added to offset
    uint32_t thr;                       // 0: nothing is dropped; 65536: everything is
    float scale;
};

inline bool drop_p_ok(double p) { return p >= 0. && p <= 1.; }      // NaN: no
inline DropKey drop_key(double p, unsigned long long seed, unsigned long long offset, const unsigned long long* step) {
    DropKey k;
    k.k0 = (uint32_t)seed;
    k.k1 = (uint32_t)(seed >> 32);
    k.offset = offset;
    k.step = step;
    k.thr = (uint32_t)floor(p * 65536. + 0.5);
    k.scale = k.thr >= 65536u ? 0.f : (float)(65536. / (65536. - k.thr));
    return k;
}

__device__ __forceinline__ unsigned long long drop_offset(const DropKey& k) { return k.step ? k.offset + *k.step : k.offset; }

__device__ __forceinline__ uint4 drop_words(const DropKey& k, unsigned long long offset, unsigned long long counter) {
    uint32_t c0 = (uint32_t)counter, c1 = (uint32_t)(counter >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = k.k0, k1 = k.k1;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long a = (unsigned long long)0xD2511F53u * c0, b = (unsigned long long)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}
// is the element with index i (0 .. 7) of a counter kept?
__device__ __forceinline__ bool drop_keep(const uint4& w, int i, uint32_t thr) {
    const uint32_t u = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
    return ((i & 1) ? u >> 16 : u & 0xFFFFu) >= thr;
}
// the same for one element by its number
__device__ __forceinline__ bool drop_keep_at(const DropKey& k, unsigned long long offset, unsigned long long e) {
    const uint4 w = drop_words(k, offset, e >> 3);
    return drop_keep(w, (int)(e & 7), k.thr);
}

}  // namespace dr
