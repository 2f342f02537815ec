// What the attention kernels share: the split of the work, the partial results of a split cache, masks and softmax pieces.
//
// For query row (t, head) at position p, with z_j = scale q.k_j over the visible positions j:
//   m = max z, l = sum e^(z_j - m), out = sum e^(z_j - m) v_j / l, lse = m + ln l;
// the maximum and the sum run along, so scores are never stored, and parts of a cache that were worked on apart are joined by
// rescaling them to the common maximum.  Everything is kept in powers of two: z carries log2 e.
//
// A row block is a run of rows r = i * G + g of one cached head: query i of the sequence, head g of the G query heads that read that
// cached head, so that a key or value read once serves all of them.
#pragma once
#include "common.hpp"

namespace qarl {

typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) const char *LdsPtr;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
constexpr float kNegInf = -__builtin_inff();
constexpr float kStale = 8.f;   // a running maximum may lag behind by this many powers of two before the sums are rescaled

// How a call is split: each kernel takes the sequences whose row count (queries times G) lies on its side of few_rows, and cuts a
// sequence's cache into pieces of `chunk` positions.
struct AttnPlan {
    int few_nr;        // the kernel for few rows: 16 * few_nr rows at a time; 0: not launched
    int few_chunk, few_splits;
    int tile;          // the kernel for many rows is launched
    int tile_chunk, tile_splits, tile_blocks;   // tile_blocks: bound of the row blocks of one cached head
    int splits;        // room for partial results per row (0: none)
};

constexpr int kFewTile = 32;      // positions a wavefront of the few-row kernel takes at a time
constexpr int kManyTile = 64;     // positions of a tile of the many-row kernel
constexpr int kManyWaves = 8, kManyRows = 256;

// Partial results in the workspace: O [splits][T * q_heads][D], then (m, l) [splits][T * q_heads], then the number of pieces [T * q_heads]
struct AttnParts {
    float *o;
    float *ml;
    int32_t *count;
    int splits;
    int64_t rows;
};

struct SeqRange {
    int row_lo, n;        // first query row, queries
    int kv;               // cached positions, as the caller gives them: query i stands at kv - n + i
    int cap;              // positions from here on do not exist
};

__device__ __forceinline__ SeqRange seq_range(const AttnArgs &a, int s)
{
    SeqRange r;
    const int lo = max(0, min(a.T, a.q_offsets[s])), hi = max(0, min(a.T, a.q_offsets[s + 1]));
    r.row_lo = lo;
    r.n = max(0, hi - lo);
    r.kv = max(0, a.kv_lens[s]);
    const int64_t table = (int64_t)a.table_width << a.kv.page_shift;
    r.cap = (int)min((int64_t)min(r.kv, a.max_kv_len), table);
    return r;
}

// Positions [begin, end) that queries [i0, i1] see between them (none: begin == end)
__device__ __forceinline__ void visible_range(const AttnArgs &a, const SeqRange &s, int i0, int i1, int &begin, int &end)
{
    const int64_t p0 = (int64_t)s.kv - s.n + i0, p1 = (int64_t)s.kv - s.n + i1;
    const int64_t e = min(p1 + 1, (int64_t)s.cap);
    const int64_t b = a.window > 0 ? max((int64_t)0, p0 - a.window + 1) : 0;
    end = (int)max((int64_t)0, e);
    begin = (int)min(b, (int64_t)end);
}

// What a row sees: positions lo <= j <= hi
__device__ __forceinline__ void row_bounds(const AttnArgs &a, const SeqRange &s, int i, int &lo, int &hi)
{
    const int64_t p = (int64_t)s.kv - s.n + i;
    hi = (int)min(p, (int64_t)s.cap - 1);
    lo = a.window > 0 ? (int)max((int64_t)0, p - a.window + 1) : 0;
}

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
