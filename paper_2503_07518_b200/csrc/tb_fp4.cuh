// The 4-bit row format (TB_FP4): a token's K and V rows of one KV head in 144 bytes.
//
//   bytes 0..63    K codes, channel 2 i in the low and 2 i + 1 in the high half of byte i
//   bytes 64..71   K scales, one per block of 16 channels       bytes 72..79   V scales
//   bytes 80..143  V codes
//
// An element is code x scale.  Codes are 4-bit floats (sign, 2 exponent bits, 1 mantissa bit: 0, .5, 1, 1.5, 2, 3, 4, 6); a scale is
// an unsigned 8-bit float of 5 exponent and 3 mantissa bits, whose bits 7 places up are the same number as f16.  A product has at
// most 6 significant bits and is a multiple of 2^-18 below 61440: exact in f16 and in bf16.
// Why this one: the exponents of K and V rows differ by more than an 8-bit float with 4 exponent bits spans without a second
// scale per tensor, which a cache that grows token by token does not have; a row starts and ends on 16 bytes, so that it can
// be fetched with 16-byte copies, and always touches five 32-byte sectors, as 160 bytes would.
#pragma once

#include <cuda_fp16.h>

#include "tb_common.cuh"

namespace tb {

constexpr int kFp4Row = 144, kFp4KScales = 64, kFp4VScales = 72, kFp4VCodes = 80;
constexpr uint32_t kFp4TopScale = 226;        // 10240: six times that is still an f16
constexpr uint32_t kFp4NanScale = 255;        // a block with a value that is not finite

// The two values of each byte of w as an f16 pair, low half first (scale not applied).
__device__ __forceinline__ void fp4_unpack(uint32_t w, uint32_t& p0, uint32_t& p1, uint32_t& p2, uint32_t& p3) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(p0), "=r"(p1), "=r"(p2), "=r"(p3)
        : "r"(w));
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// Scale byte number i of w (i known at compile time) in both halves of an f16 pair.
template <int i>
__device__ __forceinline__ uint32_t fp4_scale_pair(uint32_t w) {
    return __byte_perm(w, 0u, 0x0404 | (i << 4) | (i << 12)) >> 1;
}
// Two f16 values that have at most 8 significant bits as a bf16 pair: exact.
__device__ __forceinline__ uint32_t f16x2_to_bf16x2(uint32_t h) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
    const __nv_bfloat162 v = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 32 contiguous bytes, in one access where the address allows it (`wide`: uniform over the launch).
__device__ __forceinline__ void load_32_bytes(const void* p, bool wide, uint32_t (&w)[8]) {
    if (wide) {
        asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p) : "memory");
    } else {
        const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p)), b = __ldcs(reinterpret_cast<const uint4*>(p) + 1);
        w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    }
}
__device__ __forceinline__ void store_32_bytes(void* p, bool wide, const uint32_t (&w)[8]) {
    if (wide) {
        asm volatile("st.global.v8.b32 [%8], {%0,%1,%2,%3,%4,%5,%6,%7};" ::"r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]), "l"(p) : "memory");
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// 16 bf16 values (8 words) -> 8 bytes of codes and a scale.
//
// Scale: the largest magnitude a over 6, to the nearest 8-bit float.  a has 8 significant bits and six times a midpoint between two
// scales at most 7, so a / 6 is a midpoint (5 significant bits) or differs from every one by 2^-9 of its size.  The product with a rounded
// sixth, off by less than 2^-22, is therefore first rounded to 12 bits: that puts it on the midpoint if and only if a / 6 is one.
// Codes: x / scale to the nearest code.  It is a midpoint t between two codes (3 significant bits) exactly, or x and
// t scale (8 and at most 7 bits) differ by 2^-9 of their size, that is, the quotient by at least 2^-11 from t >= 1/4.  So the product
// with an approximate reciprocal (off by less than 2^-19), rounded to a multiple of 2^-13 by adding and taking away 1536, lies on
// the midpoint if and only if the exact quotient does, and on the same side otherwise; the conversion then rounds ties to
// the even code as the format wants.  What it rounds to a zero keeps its sign, which the format does not have: taken off afterwards.
__device__ __forceinline__ void fp4_encode(const uint32_t (&w)[8], uint2& codes, uint32_t& scale) {
    uint32_t top2 = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top2 = __vmaxu2(top2, w[i] & 0x7fff7fffu);
    const uint32_t top = max(top2 & 0xffffu, top2 >> 16);
    const uint32_t u = (__float_as_uint(__uint_as_float(top << 16) * (1.f / 6.f)) + 0x800u) & 0xfffff000u;
    const float ideal = __uint_as_float(u);
    // (below 2^-14 scales are multiples of 2^-17)
    uint32_t code = ideal < 6.103515625e-05f ? (uint32_t)__float2int_rn(ideal * 131072.f)
                                             : ((u + 0x7ffffu + ((u >> 20) & 1u)) >> 20) - (112u << 3);
    code = min(max(code, 1u), kFp4TopScale);
    const float s = __half2float(__ushort_as_half((unsigned short)(code << 7)));
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(s));
    uint32_t out[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t p = w[h * 4 + i];
            y[2 * i] = __fsub_rn(fmaf(bf16_lo(p), r, 1536.f), 1536.f), y[2 * i + 1] = __fsub_rn(fmaf(bf16_hi(p), r, 1536.f), 1536.f);
        }
        asm("{\n\t.reg .b8 a, b, c, d;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
            "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
            "mov.b32 %0, {a, b, c, d};\n\t}"
            : "=r"(out[h])
            : "f"(y[0]), "f"(y[1]), "f"(y[2]), "f"(y[3]), "f"(y[4]), "f"(y[5]), "f"(y[6]), "f"(y[7]));
        const uint32_t m = out[h] & 0x77777777u;
        out[h] = m | (out[h] & ((m << 1 | m << 2 | m << 3) & 0x88888888u));
    }
    const bool finite = top <= 0x7f7fu;
    codes = finite ? make_uint2(out[0], out[1]) : make_uint2(0u, 0u);
    scale = finite ? code : kFp4NanScale;
}

}  // namespace tb
