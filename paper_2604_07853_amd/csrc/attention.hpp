// What the attention kernels share: the partial results of a split cache, masks and softmax pieces (the split itself: attention_split.hpp).
//
// For query row (t, head) at position p, with z_j = scale q.k_j over the visible positions j:
//   m = max z, l = sum e^(z_j - m), out = sum e^(z_j - m) v_j / l, lse = m + ln l;
// the maximum and the sum run along, so scores are never stored, and parts of a cache that were worked on apart are joined by
// rescaling them to the common maximum.  Everything is kept in powers of two: z carries log2 e.
//
// Scores, maxima, sums and the outputs' sums are fp32.  A probability is rounded to bf16 where it meets the values (e4m3: times the value's scale): the matrix
// instructions take bf16, and the low halves would take the second product once more.  The roundings are of either sign and average out: outputs in fp32
// are 0.8e-4 (one token, 18432 positions) to 4.2e-4 (prompts of 2048) from 64 bits in the 2-norm, where rounding the exact result to bf16 costs 1.65e-3.
//
// A row block is a run of rows r = i * G + g of one cached head: query i of the sequence, head g of the G query heads that read that
// cached head, so that a key or value read once serves all of them.
#pragma once
#include "attention_split.hpp"

namespace qarl {

typedef __attribute__((address_space(3))) const char *LdsPtr;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kNegInf = -__builtin_inff();
constexpr float kStale = 8.f;   // a running maximum may lag behind by this many powers of two before the sums are rescaled

// Partial results in the workspace: O [splits][T * q_heads][D], then (m, l) [splits][T * q_heads], then the number of pieces [T * q_heads]
struct AttnParts {
    float *o;
    float *ml;
    int32_t *count;
    int splits;
    int64_t rows;
};

// max(lo, min(pos, hi)) for lo <= hi
__device__ __forceinline__ int clamp_pos(int pos, int lo, int hi)
{
    int r;
    asm("v_med3_i32 %0, %1, %2, %3" : "=v"(r) : "v"(pos), "v"(lo), "v"(hi));
    return r;
}

// A word of bf16 pairs (of four e4m3 codes) with zeros for infinities and NaN (NaN)
__device__ __forceinline__ uint32_t only_finite_bf16(uint32_t w)
{
    const uint32_t bad = ((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u;     // the top bit of a half: its exponent is all ones
    return w & ~((bad - (bad >> 15)) | bad);
}
__device__ __forceinline__ uint32_t only_finite_e4m3(uint32_t w)
{
    const uint32_t bad = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;     // the top bit of a byte: its code is 0x7f or 0xff
    return w & ~((bad - (bad >> 7)) | bad);
}

// fp32 -> bf16, nearest even, two per instruction
__device__ __forceinline__ uint32_t pack2_bf16(float x, float y)
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x, y}), bf16x2));
}
__device__ __forceinline__ bf16x8 pack_bf16x8(const float (&p)[8])
{
    return __builtin_bit_cast(bf16x8, u32x4{pack2_bf16(p[0], p[1]), pack2_bf16(p[2], p[3]), pack2_bf16(p[4], p[5]), pack2_bf16(p[6], p[7])});
}

// Eight e4m3 codes -> bf16 (exact; checked for all 256 codes on gfx950)
__device__ __forceinline__ bf16x8 widen_e4m3x8(uint32_t lo, uint32_t hi)
{
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    u32x4 o;
    o[0] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    o[1] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    o[2] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    o[3] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    return __builtin_bit_cast(bf16x8, o);
}

// Four outputs of row (t, head) from a whole cache, or of one piece of it
__device__ __forceinline__ void store_out4(const AttnArgs &a, int64_t row, int D, int d, f32x4 v)
{
    if (a.out_f32) {
        *(f32x4 *)((float *)a.out + row * D + d) = v;
    } else {
        *(u32x2 *)((uint16_t *)a.out + row * D + d) = u32x2{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
    }
}

// 1 / l; a row without visible positions (l == 0) gets zeros, a NaN stays
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.f ? 0.f : 1.0f / l; }

int launch_attention_few(const AttnArgs &a, const AttnPlan &p, const AttnParts &parts, hipStream_t s);
int launch_attention_tile(const AttnArgs &a, const AttnPlan &p, const AttnParts &parts, hipStream_t s);

}  // namespace qarl
