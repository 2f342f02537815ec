// Rotary positions of queries and keys, and their append to the paged cache with the rotation on the way.
// Bound by memory: an element is read and written once.  A workgroup takes a few tokens: its threads make the tokens' cosines and sines once, in LDS; then each
// keeps those of its eight pairs in registers and goes over the token's heads, sixteen elements a time.
#include "rope.hpp"

namespace qarl {

constexpr int kRotThreads = 256, kRotTokens = 8;

// What a thread does: the token (of the workgroup's) and the sixteen of a head that are its own, the heads it starts with and steps by
struct RotShare {
    int t, c, head, step;
    bool any;
};
__device__ __forceinline__ RotShare rot_share(int per_head, int tokens)
{
    const int rows = kRotThreads / per_head, row = threadIdx.x / per_head, step = rows / tokens;
    RotShare s;
    s.c = threadIdx.x - row * per_head;
    s.t = row / step;
    s.head = row - s.t * step;
    s.step = step;
    s.any = row < step * tokens;
    return s;
}

__device__ __forceinline__ void make_turns(const qarl_rope &rope, const int64_t *positions, int64_t t0, int tokens, float sign, float2 *turns)
{
    const int half = rope.rotary_dim / 2;
    for (int i = threadIdx.x; i < tokens * half; i += kRotThreads) {
        const int t = i / half, j = i - t * half;
        float2 v = rope_turn(rope.turns[j], positions[t0 + t], rope.amplitude);
        v.y *= sign;
        turns[i] = v;
    }
}

template <bool F32>
__device__ __forceinline__ void load16(const void *p, const int (&at)[2], float (&x)[16])
{
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        if (F32) {
            const f32x4 a = *(const f32x4 *)((const float *)p + at[r]), b = *(const f32x4 *)((const float *)p + at[r] + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[8 * r + i] = a[i];
                x[8 * r + 4 + i] = b[i];
            }
        } else {
            const u32x4 w = *(const u32x4 *)((const uint16_t *)p + at[r]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[8 * r + 2 * i] = __uint_as_float(w[i] << 16);
                x[8 * r + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        }
    }
}

template <bool F32>
__device__ __forceinline__ void store16(void *p, const int (&at)[2], const float (&x)[16])
{
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        if (F32) {
            *(f32x4 *)((float *)p + at[r]) = f32x4{x[8 * r], x[8 * r + 1], x[8 * r + 2], x[8 * r + 3]};
            *(f32x4 *)((float *)p + at[r] + 4) = f32x4{x[8 * r + 4], x[8 * r + 5], x[8 * r + 6], x[8 * r + 7]};
        } else {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[8 * r + i];
            *(u32x4 *)((uint16_t *)p + at[r]) = f32_to_bf16x8(y);
        }
    }
}

template <bool F32>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a, int tokens)
{
    extern __shared__ float2 turns[];
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int rot = a.rope.rotary_dim, half = rot / 2, layout = a.rope.layout;
    make_turns(a.rope, a.positions, t0, (int)min((int64_t)tokens, a.T - t0), a.inverse ? -1.f : 1.f, turns);
    __syncthreads();
    const RotShare s = rot_share(a.head_dim / 16, tokens);
    if (!s.any || t0 + s.t >= a.T) return;
    const RopeRuns runs = rope_runs(s.c, rot, layout);
    float2 turn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i] = runs.turned ? turns[s.t * half + 8 * s.c + i] : make_float2(1.f, 0.f);
    constexpr int kSize = F32 ? 4 : 2;
    for (int h = s.head; h < a.q.heads + a.k.heads; h += s.step) {
        const bool key = h >= a.q.heads;
        const int64_t head = key ? h - a.q.heads : h;
        const char *in = (const char *)(key ? a.k.in : a.q.in);
        char *out = (char *)(key ? a.k.out : a.q.out);
        const int64_t from = (t0 + s.t) * (key ? a.k.token_stride : a.q.token_stride) + head * (key ? a.k.head_stride : a.q.head_stride);
        const int64_t to = (t0 + s.t) * (key ? a.k.out_token_stride : a.q.out_token_stride) + head * (key ? a.k.out_head_stride : a.q.out_head_stride);
        float v[16];
        load16<F32>(in + from * kSize, runs.at, v);
        if (runs.turned) rope_apply(v, turn, layout);
        store16<F32>(out + to * kSize, runs.at, v);
    }
}

static int rot_tokens(int64_t T, int per_head)
{
    int tokens = kRotTokens;
    while (tokens > 1 && (tokens > kRotThreads / per_head || (T + tokens - 1) / tokens < 1024)) tokens /= 2;
    return tokens;
}

int launch_rotary(const RotaryArgs &a, hipStream_t s)
{
    const int tokens = rot_tokens(a.T, a.head_dim / 16);
    const int64_t blocks = (a.T + tokens - 1) / tokens;
    if (blocks > 0x7fffffffLL) {
        set_error("qarl_rotary: %lld tokens exceed the grid limit", (long long)a.T);
        return QARL_ERR_UNSUPPORTED;
    }
    const size_t lds = (size_t)tokens * (a.rope.rotary_dim / 2) * sizeof(float2);
    if (a.f32) rotary_kernel<true><<<dim3((unsigned)blocks), dim3(kRotThreads), lds, s>>>(a, tokens);
    else rotary_kernel<false><<<dim3((unsigned)blocks), dim3(kRotThreads), lds, s>>>(a, tokens);
    return check_hip(hipGetLastError(), "rotary_kernel");
}

// ---- the append: queries as above; keys turned and written into the cache, values written.  The lanes of a head (four or eight) stand side by side in a
// wavefront, which is all that the quantizers need to know of one another; what they quantize are the turned fp32 values.
template <int D, int FMT>
__global__ __launch_bounds__(kRotThreads) void rotary_write_kernel(RotaryWriteArgs a, int tokens)
{
    constexpr int kLanes = D / 16;
    extern __shared__ float2 turns[];
    // e2m1: a head's turned values, back in their order for its groups
    __shared__ float ordered[FMT == QARL_KV_E2M1 ? kRotThreads * 16 : 1];
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int rot = a.rope.rotary_dim, half = rot / 2, layout = a.rope.layout;
    make_turns(a.rope, a.positions, t0, (int)min((int64_t)tokens, a.T - t0), 1.f, turns);
    __syncthreads();
    const RotShare s = rot_share(kLanes, tokens);
    const int64_t token = t0 + s.t;
    if (!s.any || token >= a.T) return;
    const RopeRuns runs = rope_runs(s.c, rot, layout);
    const int straight[2] = {16 * s.c, 16 * s.c + 8};
    float2 turn[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) turn[i] = runs.turned ? turns[s.t * half + 8 * s.c + i] : make_float2(1.f, 0.f);
    const KvArgs &kv = a.kv;
    const int64_t slot = a.slots[token];
    const bool live = slot >= 0 && slot < ((int64_t)kv.num_pages << kv.page_shift);
    const int64_t page = slot >> kv.page_shift, in_page = slot & ((1 << kv.page_shift) - 1);
    for (int h = s.head; h < a.q.heads + 2 * kv.kv_heads; h += s.step) {
        float v[16];
        if (h < a.q.heads) {
            load16<false>((const uint16_t *)a.q.in + token * a.q.token_stride + h * a.q.head_stride, runs.at, v);
            if (runs.turned) rope_apply(v, turn, layout);
            store16<false>((uint16_t *)a.q.out + token * a.q.out_token_stride + h * a.q.out_head_stride, runs.at, v);
            continue;
        }
        if (!live) break;
        const bool key = h < a.q.heads + kv.kv_heads;
        const int head = h - a.q.heads - (key ? 0 : kv.kv_heads);
        const int64_t row = ((page * kv.kv_heads + head) << kv.page_shift) + in_page;
        int at[2] = {key ? runs.at[0] : straight[0], key ? runs.at[1] : straight[1]};
        load16<false>(key ? (const uint16_t *)a.k + token * a.k_token_stride + head * a.k_head_stride
                          : (const uint16_t *)a.v + token * a.v_token_stride + head * a.v_head_stride, at, v);
        if (key && runs.turned) rope_apply(v, turn, layout);
        void *to = key ? kv.k : kv.v, *scales = key ? kv.k_scales : kv.v_scales;
        if (FMT == QARL_KV_BF16) {
            store16<false>((uint16_t *)to + row * D, at, v);
        } else if (FMT == QARL_KV_E4M3) {
            float run[2][8], absmax = 0.f;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int i = 0; i < 8; ++i) run[r][i] = v[8 * r + i];
                absmax = LaneScale::absmax8(run[r], absmax);
            }
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) absmax = fmaxf(absmax, __shfl_xor(absmax, o, 64));
            const LaneScale sc(absmax);
#pragma unroll
            for (int r = 0; r < 2; ++r) *(u32x2 *)((uint8_t *)to + row * D + at[r]) = sc.quantize8(run[r]);
            if (s.c == 0) ((float *)scales)[row] = sc.stored();
        } else {
            if (key) {
                float *mine = ordered + (threadIdx.x - s.c) * 16;      // this head's place
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < 8; i += 4)
                        *(f32x4 *)(mine + at[r] + i) = f32x4{v[8 * r + i], v[8 * r + i + 1], v[8 * r + i + 2], v[8 * r + i + 3]};
                __builtin_amdgcn_wave_barrier();
                asm volatile("" ::: "memory");      // (the lanes of a head write and read in the order of their wavefront)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const f32x4 w = *(const f32x4 *)(mine + straight[0] + i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[i + e] = w[e];
                }
                __builtin_amdgcn_wave_barrier();
                asm volatile("" ::: "memory");
            }
            float run[2][8], absmax = 0.f;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int i = 0; i < 8; ++i) run[r][i] = v[8 * r + i];
                absmax = LaneScale::absmax8(run[r], absmax);
            }
            if (D == 128) absmax = fmaxf(absmax, __shfl_xor(absmax, 1, 64));
            const E2m1Scale sc(absmax);
            *(u32x2 *)((uint8_t *)to + row * (D / 2) + 8 * s.c) = u32x2{sc.quantize8(run[0]), sc.quantize8(run[1])};
            if (D == 64 || (s.c & 1) == 0) ((uint8_t *)scales)[row * 4 + s.c * 16 / (D / 4)] = sc.byte;
        }
    }
}

int launch_rotary_write(const RotaryWriteArgs &a, hipStream_t s)
{
    const int D = a.kv.head_dim, tokens = rot_tokens(a.T, D / 16);
    const int64_t blocks = (a.T + tokens - 1) / tokens;
    if (blocks > 0x7fffffffLL) {
        set_error("qarl_rotary_kv_write: %lld tokens exceed the grid limit", (long long)a.T);
        return QARL_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)blocks), block(kRotThreads);
    const size_t lds = (size_t)tokens * (a.rope.rotary_dim / 2) * sizeof(float2);
    const int fmt = a.kv.fmt;
    if (D == 128) {
        if (fmt == QARL_KV_BF16) rotary_write_kernel<128, QARL_KV_BF16><<<grid, block, lds, s>>>(a, tokens);
        else if (fmt == QARL_KV_E4M3) rotary_write_kernel<128, QARL_KV_E4M3><<<grid, block, lds, s>>>(a, tokens);
        else rotary_write_kernel<128, QARL_KV_E2M1><<<grid, block, lds, s>>>(a, tokens);
    } else {
        if (fmt == QARL_KV_BF16) rotary_write_kernel<64, QARL_KV_BF16><<<grid, block, lds, s>>>(a, tokens);
        else if (fmt == QARL_KV_E4M3) rotary_write_kernel<64, QARL_KV_E4M3><<<grid, block, lds, s>>>(a, tokens);
        else rotary_write_kernel<64, QARL_KV_E2M1><<<grid, block, lds, s>>>(a, tokens);
    }
    return check_hip(hipGetLastError(), "rotary_write_kernel");
}

}  // namespace qarl
