// The 4-bit cache: offsets and the row quantiser.
//
// A row x of 128 bf16 values is held as unsigned codes u with a scale s and an offset z:
//   z = min x (exact in bf16),  s = bf16((max x - z) / 15),  u_d = clamp(rne((x_d - z) / s), 0, 15),  value z + u s.
// Byte i of a row's 64 bytes holds dim i in its low and dim 64 + i in its high four bits, so that one mask leaves four
// dims that lie side by side.  Scale and offset share a 32-bit word (scale low).
#pragma once
#include "slim_common.cuh"
#include "slim_quant.cuh"

namespace slim {

constexpr int kRow4Bytes = kHeadDim / 2;

__host__ __device__ inline size_t code4_block_offset(int page, int head, int kv, int Hkv)
{
    return ((size_t)((size_t)page * Hkv + head) * 2 + kv) * (size_t)(kPageTokens * kRow4Bytes);
}

__device__ __forceinline__ float pair_scale(uint32_t pair) { return __uint_as_float(pair << 16); }
__device__ __forceinline__ float pair_offset(uint32_t pair) { return __uint_as_float(pair & 0xFFFF0000u); }

__device__ __forceinline__ uint32_t q4_min_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.bf16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Scale and offset of a row whose smallest and largest value are lo and hi, as the cache holds them.
__device__ __forceinline__ uint32_t q4_pair(float lo, float hi)
{
    const float s = __fdiv_rn(hi - lo, 15.f);
    const __nv_bfloat162 p = __floats2bfloat162_rn(s, lo);
    return *reinterpret_cast<const uint32_t *>(&p);
}

// What the codes of a row are formed with.  The quotient (x - z) / s is the correctly rounded one: p = d * rc with
// rc = RN(1 / s), its exact residual r = d - s p by a fused multiply-add, q = p + r rc (Markstein's correction).  A scale
// outside [2^-60, 2^60] is brought to the middle of the range together with the differences, by an exact power of two.
struct Q4Row {
    float z, f, ns, rc;
    __device__ __forceinline__ explicit Q4Row(uint32_t pair)
    {
        const float s = pair_scale(pair);
        z = pair_offset(pair);
        f = 1.f;
        if (s < 0x1p-60f) f = 0x1p100f;
        else if (s > 0x1p60f) f = 0x1p-100f;
        const float ss = s * f;
        ns = -ss;
        rc = (s > 0.f) ? __frcp_rn(ss) : 0.f;
    }
    // 0x4B400000 + round((x - z) / s) of two values, not yet clamped to 15
    __device__ __forceinline__ void codes(float x0, float x1, uint32_t &u0, uint32_t &u1) const
    {
        const uint64_t d2 = ap_mul2(ap_add2(ap_pack(x0, x1), ap_pack(-z, -z)), ap_pack(f, f));
        const uint64_t rc2 = ap_pack(rc, rc), p2 = ap_mul2(d2, rc2);
        const uint64_t q2 = ap_fma2(ap_fma2(ap_pack(ns, ns), p2, d2), rc2, p2);
        const uint64_t t2 = ap_add2(q2, ap_pack(kRoundMagic, kRoundMagic));
        u0 = min((uint32_t)t2, 0x4B40000Fu);
        u1 = min((uint32_t)(t2 >> 32), 0x4B40000Fu);
    }
    // four values (two words of bf16 pairs): a code in every byte
    __device__ __forceinline__ uint32_t codes4(uint32_t a, uint32_t b) const
    {
        uint32_t u0, u1, u2, u3;
        codes(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u), u0, u1);
        codes(__uint_as_float(b << 16), __uint_as_float(b & 0xFFFF0000u), u2, u3);
        return __byte_perm(__byte_perm(u0, u1, 0x0040), __byte_perm(u2, u3, 0x0040), 0x5410);
    }
};

}  // namespace slim
