// Rotary positions of queries and keys, and their append to the paged cache with the rotation on the way.
// Bound by memory: an element is read and written once.  A workgroup takes a few tokens: its threads make the tokens' cosines and sines once, in LDS; then each
// keeps those of its pairs in registers (eight of 16-bit elements, four of 32) and goes over the token's heads, two runs of 16 bytes a time.
// 16384 tokens of 32 + 4 heads of 128 in bf16, 302 MB: 57.1 us, 5.3 TB/s (cached accesses 64); 1733 of 28 + 4 in fp32, 57 MB, which the last-level cache holds: 9.8 us.
// With the append: 16384 tokens to a bf16 cache, 336 MB: 64.6 us, 5.2 TB/s; 256 to an e4m3 one 6.1 us, of which 4 are any launch's.
#include "rope.hpp"

namespace qarl {

constexpr int kRotThreads = 256, kRotTokens = 8;
constexpr int64_t kRotCached = (int64_t)64 << 20;     // calls that move more pass the caches

// What a thread does: the token (of the workgroup's) and the lane of a head that it is, the heads it starts with and steps by
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

// 2 E elements at two places, 16 bytes each: as they are, and as numbers
struct Raw {
    u32x4 w[2];
};
template <int E, bool NT>
__device__ __forceinline__ Raw load_raw(const void *p, const int (&at)[2])
{
    return Raw{{load_as<NT, u32x4>((const char *)p + at[0] * (16 / E)), load_as<NT, u32x4>((const char *)p + at[1] * (16 / E))}};
}
template <int E>
__device__ __forceinline__ void numbers(const Raw &r, float (&x)[2 * E])
{
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < E; ++i)
            x[E * k + i] = E == 4 ? __uint_as_float(r.w[k][i]) : __uint_as_float(i & 1 ? r.w[k][i >> 1] & 0xffff0000u : r.w[k][i >> 1] << 16);
}
template <int E, bool NT>
__device__ __forceinline__ void store_runs(void *p, const int (&at)[2], const float (&x)[2 * E])
{
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        u32x4 w;
        if (E == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(x[E * k + (i & (E - 1))]);
        } else {
            float y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = x[E * k + (i & (E - 1))];
            w = f32_to_bf16x8(y);
        }
        store_as<NT>((char *)p + at[k] * (16 / E), w);
    }
}

template <bool F32, bool NT>
__global__ __launch_bounds__(kRotThreads) void rotary_kernel(RotaryArgs a, int tokens)
{
    constexpr int E = F32 ? 4 : 8, kSize = F32 ? 4 : 2;
    extern __shared__ float2 turns[];
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int rot = a.rope.rotary_dim, layout = a.rope.layout;
    const RotShare s = rot_share(a.head_dim / (2 * E), tokens);
    const RopeRuns runs = rope_runs<E>(s.c, a.head_dim, rot, layout);
    const int64_t token = t0 + s.t;
    const int heads = s.any && token < a.T ? a.q.heads + a.k.heads : 0;
    const auto from = [&](int h) {
        const bool key = h >= a.q.heads;
        return (const char *)(key ? a.k.in : a.q.in) +
               (token * (key ? a.k.token_stride : a.q.token_stride) + (key ? h - a.q.heads : h) * (key ? a.k.head_stride : a.q.head_stride)) * kSize;
    };
    // the first head's values are requested before the angles are made
    Raw raw = {};
    if (s.head < heads) raw = load_raw<E, NT>(from(s.head), runs.at);
    make_turns(a.rope, a.positions, t0, (int)min((int64_t)tokens, a.T - t0), a.inverse ? -1.f : 1.f, turns);
    __syncthreads();
    if (heads == 0) return;
    float2 turn[E];
    rope_turns<E>(turns + s.t * (rot / 2), runs, layout, turn);
    for (int h = s.head; h < heads; h += s.step) {
        float v[2 * E];
        numbers<E>(raw, v);
        if (h + s.step < heads) raw = load_raw<E, NT>(from(h + s.step), runs.at);
        if (runs.turned) rope_apply<E>(v, turn, layout);
        const bool key = h >= a.q.heads;
        store_runs<E, NT>((char *)(key ? a.k.out : a.q.out) +
                          (token * (key ? a.k.out_token_stride : a.q.out_token_stride) + (key ? h - a.q.heads : h) * (key ? a.k.out_head_stride : a.q.out_head_stride)) * kSize,
                      runs.at, v);
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
    const int tokens = rot_tokens(a.T, a.head_dim / (a.f32 ? 8 : 16));
    const int64_t blocks = (a.T + tokens - 1) / tokens;
    if (blocks > 0x7fffffffLL) {
        set_error("qarl_rotary: %lld tokens exceed the grid limit", (long long)a.T);
        return QARL_ERR_UNSUPPORTED;
    }
    const size_t lds = (size_t)tokens * (a.rope.rotary_dim / 2) * sizeof(float2);
    const dim3 grid((unsigned)blocks), block(kRotThreads);
    const bool nt = a.T * (a.q.heads + a.k.heads) * a.head_dim * (a.f32 ? 8 : 4) > kRotCached;
    if (a.f32) {
        if (nt) rotary_kernel<true, true><<<grid, block, lds, s>>>(a, tokens);
        else rotary_kernel<true, false><<<grid, block, lds, s>>>(a, tokens);
    } else {
        if (nt) rotary_kernel<false, true><<<grid, block, lds, s>>>(a, tokens);
        else rotary_kernel<false, false><<<grid, block, lds, s>>>(a, tokens);
    }
    return check_hip(hipGetLastError(), "rotary_kernel");
}

// ---- the append: queries as above; keys turned and written into the cache, values written.  The lanes of a head (four or eight) stand side by side in a
// wavefront, which is all that the quantizers need to know of one another; what they quantize are the turned fp32 values.
template <int D, int FMT, bool NT>
__global__ __launch_bounds__(kRotThreads) void rotary_write_kernel(RotaryWriteArgs a, int tokens)
{
    constexpr int kLanes = D / 16, E = 8;
    extern __shared__ float2 turns[];
    // e2m1: a head's turned values, back in their order for its groups
    __shared__ float ordered[FMT == QARL_KV_E2M1 ? kRotThreads * 16 : 1];
    const int64_t t0 = (int64_t)blockIdx.x * tokens;
    const int rot = a.rope.rotary_dim, layout = a.rope.layout;
    const RotShare s = rot_share(kLanes, tokens);
    const int64_t token = t0 + s.t;
    const KvArgs &kv = a.kv;
    const int q_heads = a.q.heads, heads = s.any && token < a.T ? q_heads + 2 * kv.kv_heads : 0;
    const RopeRuns runs = rope_runs<E>(s.c, D, rot, layout);
    const int plain[2] = {FMT == QARL_KV_E2M1 ? 16 * s.c : 8 * s.c, FMT == QARL_KV_E2M1 ? 16 * s.c + 8 : D / 2 + 8 * s.c};     // of a value's head
    const auto load = [&](int h) {
        if (h < q_heads) return load_raw<E, NT>((const uint16_t *)a.q.in + token * a.q.token_stride + h * a.q.head_stride, runs.at);
        if (h < q_heads + kv.kv_heads) return load_raw<E, NT>((const uint16_t *)a.k + token * a.k_token_stride + (h - q_heads) * a.k_head_stride, runs.at);
        return load_raw<E, NT>((const uint16_t *)a.v + token * a.v_token_stride + (h - q_heads - kv.kv_heads) * a.v_head_stride, plain);
    };
    // the first head's values and the slot are requested before the angles are made
    Raw raw = {};
    int64_t slot = -1;
    if (s.head < heads) {
        raw = load(s.head);
        slot = a.slots[token];
    }
    make_turns(a.rope, a.positions, t0, (int)min((int64_t)tokens, a.T - t0), 1.f, turns);
    __syncthreads();
    if (heads == 0) return;
    float2 turn[E];
    rope_turns<E>(turns + s.t * (rot / 2), runs, layout, turn);
    const bool live = slot >= 0 && slot < ((int64_t)kv.num_pages << kv.page_shift);
    const int64_t page = slot >> kv.page_shift, in_page = slot & ((1 << kv.page_shift) - 1);
    for (int h = s.head; h < heads; h += s.step) {
        float v[16];
        numbers<E>(raw, v);
        if (h + s.step < heads) raw = load(h + s.step);
        if (h < q_heads) {
            if (runs.turned) rope_apply<E>(v, turn, layout);
            store_runs<E, NT>((uint16_t *)a.q.out + token * a.q.out_token_stride + h * a.q.out_head_stride, runs.at, v);
            continue;
        }
        if (!live) break;
        const bool key = h < q_heads + kv.kv_heads;
        const int64_t row = ((page * kv.kv_heads + (h - q_heads - (key ? 0 : kv.kv_heads))) << kv.page_shift) + in_page;
        const int at[2] = {key ? runs.at[0] : plain[0], key ? runs.at[1] : plain[1]};
        if (key && runs.turned) rope_apply<E>(v, turn, layout);
        void *to = key ? kv.k : kv.v, *scales = key ? kv.k_scales : kv.v_scales;
        if (FMT == QARL_KV_BF16) {
            store_runs<E, NT>((uint16_t *)to + row * D, at, v);
            continue;
        }
        if (FMT == QARL_KV_E2M1 && key) {
            float *mine = ordered + (threadIdx.x - s.c) * 16;      // this head's place
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < 8; i += 4) *(f32x4 *)(mine + at[r] + i) = f32x4{v[8 * r + i], v[8 * r + i + 1], v[8 * r + i + 2], v[8 * r + i + 3]};
            __builtin_amdgcn_wave_barrier();
            asm volatile("" ::: "memory");      // (the lanes of a head write and read in the order of their wavefront)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                const f32x4 w = *(const f32x4 *)(mine + 16 * s.c + i);
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
        if (FMT == QARL_KV_E4M3) {
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) absmax = fmaxf(absmax, __shfl_xor(absmax, o, 64));
            const LaneScale sc(absmax);
#pragma unroll
            for (int r = 0; r < 2; ++r) *(u32x2 *)((uint8_t *)to + row * D + at[r]) = sc.quantize8(run[r]);
            if (s.c == 0) ((float *)scales)[row] = sc.stored();
        } else {
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
    const bool nt = a.T * (a.q.heads + a.kv.kv_heads) * D * 4 > kRotCached;
#define QARL_ROT_WRITE(D, FMT) \
    if (nt) rotary_write_kernel<D, FMT, true><<<grid, block, lds, s>>>(a, tokens); \
    else rotary_write_kernel<D, FMT, false><<<grid, block, lds, s>>>(a, tokens)
#define QARL_ROT_WRITE_TO(D) \
    if (a.kv.fmt == QARL_KV_BF16) { \
        QARL_ROT_WRITE(D, QARL_KV_BF16); \
    } else if (a.kv.fmt == QARL_KV_E4M3) { \
        QARL_ROT_WRITE(D, QARL_KV_E4M3); \
    } else { \
        QARL_ROT_WRITE(D, QARL_KV_E2M1); \
    }
    if (D == 128) {
        QARL_ROT_WRITE_TO(128)
    } else {
        QARL_ROT_WRITE_TO(64)
    }
#undef QARL_ROT_WRITE_TO
#undef QARL_ROT_WRITE
    return check_hip(hipGetLastError(), "rotary_write_kernel");
}

}  // namespace qarl
