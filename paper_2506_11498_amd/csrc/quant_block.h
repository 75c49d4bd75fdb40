// Codes of 8 bits with a scale per block of rows and KV head: the arithmetic shared by the kernels that write, read and
// attend over such a cache.
//
//   scale  s = 2^e, the least e >= -120 with max |x| over the block <= Q 2^e; Q = 127 (int8) or 448 (e4m3)
//   code   c = round(x / s), ties to even: a whole number in [-127, 127], or the nearest e4m3 number (4 bits exponent of
//          bias 7, 3 bits fraction, no infinities)
//   value  c s
// Magnitudes above 127 * 2^121 (int8) or 240 * 2^120 (e4m3), the largest values that are numbers of 32 bits, count as these: the next code's
// or the next scale's value would be 2^128.
// Because s is a power of two, x / s is exact, so the code is that of the definition bit for bit; c has at most 8
// significant bits, so the value is exact in bf16; and a code that moves to a block of another scale keeps its value unless
// the new scale is too coarse for it (int8: some low bits; e4m3: subnormals only).  With s = max / Q the values would be
// up to twice as fine for int8, and every move of a row would round it again.
#pragma once
#include "common.h"

namespace lrsa {

constexpr int QUANT_INT8 = 0, QUANT_E4M3 = 1;
constexpr int QUANT_MAX_BLOCK = 128;

// A cache of 8 bits: K and V codes by the same strides (bytes), scales [B, Hkv, nb] of each
struct QuantDims {
    int fmt, block, log_block, nb;
    int64_t st[3];
    uint8_t *K, *V;
    float *Ks, *Vs;
};

#if defined(__HIPCC__)
template <int FMT> constexpr float QUANT_LARGEST = FMT == QUANT_INT8 ? 0x1.fcp127f : 0x1.ep127f;
template <int FMT>
__device__ __forceinline__ float quant_scale(float top) {
    constexpr int UP = FMT == QUANT_INT8 ? 6 : 8;                             // Q = 1.984375 * 2^6, 1.75 * 2^8
    constexpr uint32_t FRAC = FMT == QUANT_INT8 ? 0x7e0000u : 0x600000u;
    const uint32_t u = __float_as_uint(fminf(top, QUANT_LARGEST<FMT>));
    const int e = max(int(u >> 23) - UP + ((u & 0x7fffffu) > FRAC ? 1 : 0), 127 - 120);
    return __uint_as_float(uint32_t(e) << 23);
}

// Keeps the compiler from taking codes apart before they are used, or from keeping them so afterwards: as floats they take four times the
// registers (k_decode_quant spilled, k_evict_quant ran two workgroups per CU).
__device__ __forceinline__ uint32_t as_loaded(uint32_t w) {
    asm("" : "+v"(w));
    return w;
}

// 8 codes -> their whole or e4m3 numbers
template <int FMT>
__device__ __forceinline__ void code_values(uint2 c, float (&v)[8]) {
    const uint32_t w[2] = {c.x, c.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (FMT == QUANT_INT8) {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[4 * i + j] = float(int8_t(w[i] >> (8 * j)));
        } else {
            typedef float f32x2 __attribute__((ext_vector_type(2)));
            const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(int(w[i]), false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(int(w[i]), true);
            v[4 * i] = lo.x; v[4 * i + 1] = lo.y; v[4 * i + 2] = hi.x; v[4 * i + 3] = hi.y;
        }
    }
}
// 8 values times `inv`, none beyond the largest code -> codes.  What is infinite or no number gets some finite code (int8 by what the
// sum's low byte is, e4m3 by the clamp): a row that a token does not see then has no part in its output, 0 * code being 0.
template <int FMT>
__device__ __forceinline__ uint2 make_codes(const float (&v)[8], float inv) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (FMT == QUANT_INT8) {
            // 1.5 * 2^23 + x: numbers there are 1 apart, so the sum is rounded as wanted and its low byte is the code
            uint32_t x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = __float_as_uint(__builtin_fmaf(v[4 * i + j], inv, 12582912.0f));
            w[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(x[3], x[2], 0x0c0c0400u), __builtin_amdgcn_perm(x[1], x[0], 0x0c0c0400u), 0x05040100u);
        } else {
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = __builtin_amdgcn_fmed3f(v[4 * i + j] * inv, -448.0f, 448.0f);
            const int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
            w[i] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], c, true));
        }
    }
    return uint2{w[0], w[1]};
}

// Reads and writes past the caches, of rows that are touched once
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 stream_load(const void* p) {
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    return uint4{v.x, v.y, v.z, v.w};
}
__device__ __forceinline__ void stream_store(void* p, const uint4& v) { __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4*>(p)); }

// 8 neighbouring elements of a row
__device__ __forceinline__ void load8(const bf16_t* p, float (&v)[8]) { Elem<bf16_t>::load(p, v); }
__device__ __forceinline__ void stream_load8(const bf16_t* p, float (&v)[8]) { Elem<bf16_t>::unpack(stream_load(p), v); }
__device__ __forceinline__ void stream_load8(const float* p, float (&v)[8]) {
    const uint4 a = stream_load(p), b = stream_load(p + 4);
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
// exact where v is a value of the cache: 8 significant bits
__device__ __forceinline__ void store8(bf16_t* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_perm(__float_as_uint(v[2 * i + 1]), __float_as_uint(v[2 * i]), 0x07060302u);
    *reinterpret_cast<uint4*>(p) = uint4{w[0], w[1], w[2], w[3]};
}
__device__ __forceinline__ void store8(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = float4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<float4*>(p)[1] = float4{v[4], v[5], v[6], v[7]};
}

// largest of the block's values; every thread calls; `sm` holds a float per wave
template <int NT>
__device__ __forceinline__ float block_max(float v, float* sm) {
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = v;
    __syncthreads();
    v = sm[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) v = fmaxf(v, sm[i]);
    return v;
}
#endif

}  // namespace lrsa
