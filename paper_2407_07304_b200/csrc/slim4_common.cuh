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

// (A NaN stays one: a row that holds a NaN gets it as scale and offset, and so as its values.)
__device__ __forceinline__ uint32_t q4_min_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t q4_max_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// the smaller (the larger) value of a pair
__device__ __forceinline__ float q4_min_of(uint32_t a)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;\n" : "=f"(r) : "f"(__uint_as_float(a << 16)), "f"(__uint_as_float(a & 0xFFFF0000u)));
    return r;
}
__device__ __forceinline__ float q4_max_of(uint32_t a)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;\n" : "=f"(r) : "f"(__uint_as_float(a << 16)), "f"(__uint_as_float(a & 0xFFFF0000u)));
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
// rc = RN(1 / s), its exact residual r = d - s p by a fused multiply-add, q = p + r rc (Markstein's correction).  Rows whose
// scale lies outside [2^-60, 2^60] (constant rows among them, and rows with a NaN or an infinity, whose scale is one) divide
// instead: intermediates could leave the normal range there, and only a scale that is a subnormal of few bits can be so much too
// small that a quotient passes 15.5 (the others are within 2^-9: 15.06 at most).  So a code never has more than four bits.
struct Q4Row {
    uint64_t nz2, ns2, rc2;   // -z, -s and 1 / s, twice each
    uint32_t pair;
    bool far;
    __device__ __forceinline__ explicit Q4Row(uint32_t of) : pair(of)
    {
        const float s = pair_scale(pair), z = pair_offset(pair);
        far = !(s >= 0x1p-60f && s <= 0x1p60f);
        const float rc = far ? 0.f : __frcp_rn(s);
        nz2 = ap_pack(-z, -z), ns2 = ap_pack(-s, -s), rc2 = ap_pack(rc, rc);
    }
    // 0x4B400000 + the code of two values
    __device__ __forceinline__ void codes(uint32_t xx, uint32_t &u0, uint32_t &u1) const
    {
        const uint64_t d2 = ap_add2(ap_pack(__uint_as_float(xx << 16), __uint_as_float(xx & 0xFFFF0000u)), nz2);
        const uint64_t p2 = ap_mul2(d2, rc2);
        const uint64_t t2 = ap_add2(ap_fma2(ap_fma2(ns2, p2, d2), rc2, p2), ap_pack(kRoundMagic, kRoundMagic));
        u0 = (uint32_t)t2, u1 = (uint32_t)(t2 >> 32);
    }
    __device__ __noinline__ static uint32_t far_codes4(uint32_t pair, uint32_t a, uint32_t b)
    {
        const float s = pair_scale(pair), z = pair_offset(pair);
        uint32_t w = 0;
        for (int i = 0; i < 4; ++i) {
            const uint32_t xx = (i < 2) ? a : b;
            const float x = __uint_as_float((i & 1) ? (xx & 0xFFFF0000u) : (xx << 16));
            const float u = (s > 0.f) ? fminf(rintf(__fdiv_rn(x - z, s)), 15.f) : 0.f;
            w |= (uint32_t)u << (8 * i);
        }
        return w;
    }
    // four values (two words of bf16 pairs): a code in every byte
    __device__ __forceinline__ uint32_t codes4(uint32_t a, uint32_t b) const
    {
        uint32_t u0, u1, u2, u3;
        codes(a, u0, u1);
        codes(b, u2, u3);
        return __byte_perm(__byte_perm(u0, u1, 0x0040), __byte_perm(u2, u3, 0x0040), 0x5410);
    }
    // N words of codes: of the dims in lo[2 i], lo[2 i + 1] (low halves of the bytes) and those 64 further
    template <int N>
    __device__ __forceinline__ void words(const uint32_t (&lo)[2 * N], const uint32_t (&hi)[2 * N], uint32_t (&w)[N]) const
    {
        if (far) {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = far_codes4(pair, lo[2 * i], lo[2 * i + 1]) | (far_codes4(pair, hi[2 * i], hi[2 * i + 1]) << 4);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = codes4(lo[2 * i], lo[2 * i + 1]) | (codes4(hi[2 * i], hi[2 * i + 1]) << 4);
        }
    }
};

}  // namespace slim
