// The paged cache held in 4 bits, as its kernels see it, and the checks that its calls share.  Not part of the public ABI.
//
// 32 channels are 32 codes of 4 bits (E2M1) and a byte s: gfx950 converts a pair of codes to bf16 or fp32, times 2^(s - 127), in one
// instruction and exactly (all 16 codes under all 256 bytes agree with the definition; s = 255 gives NaN), and rounds a pair of fp32 to
// codes as the definition says (1,038,256 numbers, all borders between codes and their neighbours among them).
#pragma once

#include "cache.h"

namespace veda {

veda_status check_packed(const veda_packed_cache* c);
veda_cache packed_rows(const veda_packed_cache* c);                             // a cache of the same rows, for the checks of batches and row tensors
CacheArgs packed_args(const veda_packed_cache* c, const veda_cache_batch* b);   // page_b: bytes of a packed page
inline int64_t packed_head_bytes(const veda_packed_cache* c) { return (int64_t)c->page_tokens * (c->head_dim / 2 + c->head_dim / 32); }

#if defined(__HIPCC__)

constexpr uint32_t kPackedNan = 253;   // bytes from here on stand for NaN
__device__ __forceinline__ float packed_power(uint32_t s) { return __uint_as_float(s << 23); }   // 2^(s - 127) as the conversions take it; 255: NaN
__device__ __forceinline__ float packed_power_of(uint32_t s) { return packed_power(s >= kPackedNan ? 255u : s); }   // of a byte from the pool

// Eight codes, channel i in bits 4 i.. of w, as values.
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2v;
typedef __attribute__((ext_vector_type(2))) float f32x2p;
__device__ __forceinline__ uint4 packed_bf16(uint32_t w, float power) {
    uint4 x;
    x.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 0));
    x.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 1));
    x.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 2));
    x.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, power, 3));
    return x;
}
__device__ __forceinline__ void packed_f32(uint32_t w, float power, uint4 (&x)[2]) {
    const f32x2p a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, power, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, power, 1);
    const f32x2p c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, power, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, power, 3);
    x[0] = uint4{__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(b[0]), __float_as_uint(b[1])};
    x[1] = uint4{__float_as_uint(c[0]), __float_as_uint(c[1]), __float_as_uint(d[0]), __float_as_uint(d[1])};
}

// fp32 as three bf16 parts: the value with its bits cut off at 8, twice, and what is left (8 bits at most).  Only the first part of what is not finite.
__device__ __forceinline__ void packed_parts(float x, __bf16 (&p)[3]) {
    const float a = __uint_as_float(__float_as_uint(x) & 0xffff0000u), r = fabsf(x) < INFINITY ? x - a : 0.0f;
    const float b = __uint_as_float(__float_as_uint(r) & 0xffff0000u);
    p[0] = (__bf16)(fabsf(x) < INFINITY ? a : x);
    p[1] = (__bf16)b;
    p[2] = (__bf16)(r - b);
}

template <int W> __device__ __forceinline__ void packed_words(const char* p, uint32_t (&w)[W]) {
    if constexpr (W == 4) {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else if constexpr (W == 2) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        w[0] = x.x; w[1] = x.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

// bf16 rows of D channels in LDS: 16-byte chunk c of row r lies at chunk packed_chunk(c) ^ swizzle(r).  Eight neighbouring lanes write at once, in 32 banks: two
// quarters each of two rows of 128 channels, or eighths of one, or quarters of two rows of 64 (which share no banks otherwise).  Chunks half a row apart, and
// rows that are neighbours, so have to lie apart too, beside what reads want (prompts of up to 4096 tokens, window 1024: 312 us
// without a conflict; 318 with two quarters of a row in the same banks, 326 with rows as well).
template <int D> __host__ __device__ constexpr int packed_chunk(int c) { return D == 128 ? c ^ (c >> 3) * 3 : c; }
// V, for products of 16 channels: eight rows that 32 lanes read two neighbouring chunks of fall into different banks.
template <int D> __device__ __forceinline__ int packed_v_swizzle(int r) {
    const int k0 = r & 1, k1 = (r >> 1) & 1, k2 = (r >> 2) & 1;
    return D == 128 ? k2 << 3 | k0 << 2 | k1 << 1 | k0 : k2 << 2 | k1 << 1 | (k1 ^ k0);
}

#endif

}  // namespace veda
