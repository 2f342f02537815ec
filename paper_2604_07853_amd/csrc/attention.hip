// Causal attention of new tokens over the paged cache.  For query row (t, h) at position p, with z_j = scale q.k_j over the visible j:
//   m = max z, l = sum e^(z_j - m), out = sum e^(z_j - m) v_j / l, lse = m + ln l;
// the maximum and the sum run along (a block of tokens rescales what the blocks before have left), so the scores are never stored.
#include "common.hpp"

namespace qarl {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

// A wavefront per (token, query head), 64 cached tokens at a time, one per lane for the scores; for the values a lane owns
// D / 64 of the outputs.
template <int D, bool E4M3>
__global__ __launch_bounds__(256) void attention_rows_kernel(AttnArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int t = (int)(unit / a.q_heads), h = (int)(unit - (int64_t)t * a.q_heads);
    if (t >= a.T) return;
    if (t < a.q_offsets[0] || t >= a.q_offsets[a.S]) return;
    int lo = 0, hi = a.S;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.q_offsets[mid] <= t) lo = mid;
        else hi = mid;
    }
    const int n = a.q_offsets[lo + 1] - a.q_offsets[lo];
    const int64_t cap = min((int64_t)a.max_kv_len, (int64_t)a.table_width << a.kv.page_shift);
    const int p = a.kv_lens[lo] - n + (t - a.q_offsets[lo]);
    const int end = (int)min((int64_t)p + 1, cap);
    const int begin = a.window > 0 ? max(0, p - a.window + 1) : 0;
    const int kvh = h / (a.q_heads / a.kv.kv_heads);
    const uint16_t *q = (const uint16_t *)a.q + (int64_t)t * a.q_token_stride + (int64_t)h * a.q_head_stride;
    float acc[D / 64] = {};
    float m = -__builtin_inff(), l = 0.f;
    for (int j0 = begin; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        int64_t row = -1;
        float z = -__builtin_inff();
        if (j < end) {
            const int page = a.table[lo * a.table_stride + (j >> a.kv.page_shift)];
            if (page >= 0 && page < a.kv.num_pages)
                row = (((int64_t)page * a.kv.kv_heads + kvh) << a.kv.page_shift) + (j & ((1 << a.kv.page_shift) - 1));
        }
        float vs = 1.f;
        if (row >= 0) {
            float dot = 0.f;
            for (int d = 0; d < D; d += 8) {
                float qf[8], kf[8];
                bf16x8_to_f32(*(const u32x4 *)(q + d), qf);
                if (E4M3) bf16x8_to_f32(e4m3_as_bf16x8(*(const u32x2 *)((const uint8_t *)a.kv.k + row * D + d)), kf);
                else bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.kv.k + row * D + d), kf);
#pragma unroll
                for (int e = 0; e < 8; ++e) dot = fmaf(qf[e], kf[e], dot);
            }
            if (E4M3) {
                dot *= a.kv.k_scales[row];
                vs = a.kv.v_scales[row];
            }
            z = dot * (a.scale * kLog2e);
        }
        float mn = z;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) mn = fmaxf(mn, __shfl_xor(mn, o, 64));
        mn = fmaxf(mn, m);
        const float base = mn == -__builtin_inff() ? 0.f : mn;
        const float keep = exp2f(m - base);
        const float pr = row >= 0 ? exp2f(z - base) : 0.f;
        l = l * keep + wave_sum(pr);
        m = mn;
#pragma unroll
        for (int u = 0; u < D / 64; ++u) acc[u] *= keep;
        const unsigned long long some = __ballot(row >= 0);
        for (int k = 0; k < 64; ++k) {
            if (!(some >> k & 1ull)) continue;
            const int64_t rk = __shfl(row, k, 64);
            const float pk = __shfl(pr, k, 64) * __shfl(vs, k, 64);
#pragma unroll
            for (int u = 0; u < D / 64; ++u) {
                const int d = lane + 64 * u;
                float v;
                if (E4M3) v = __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)a.kv.v)[rk * D + d], 0);
                else v = bf16_bits_to_f32(((const uint16_t *)a.kv.v)[rk * D + d]);
                acc[u] = fmaf(pk, v, acc[u]);
            }
        }
    }
    const float inv = l > 0.f ? 1.0f / l : (l == l ? 0.f : l);
    const int64_t o = ((int64_t)t * a.q_heads + h) * D;
#pragma unroll
    for (int u = 0; u < D / 64; ++u) {
        if (a.out_f32) ((float *)a.out)[o + lane + 64 * u] = acc[u] * inv;
        else ((uint16_t *)a.out)[o + lane + 64 * u] = f32_to_bf16_hw(acc[u] * inv);
    }
    if (a.lse && lane == 0) a.lse[(int64_t)t * a.q_heads + h] = (m + log2f(l)) * kLn2;
}

size_t attention_ws_bytes(int T, int q_heads, int kv_heads, int head_dim, int S, int max_q_len, int max_kv_len) { return 0; }

int launch_attention(const AttnArgs &a, hipStream_t s)
{
    const int64_t units = (int64_t)a.T * a.q_heads;
    const dim3 grid((unsigned)((units + 3) / 4)), block(256);
    const bool e4m3 = a.kv.fmt == QARL_KV_E4M3;
    if (a.kv.head_dim == 128) {
        if (e4m3) attention_rows_kernel<128, true><<<grid, block, 0, s>>>(a);
        else attention_rows_kernel<128, false><<<grid, block, 0, s>>>(a);
    } else {
        if (e4m3) attention_rows_kernel<64, true><<<grid, block, 0, s>>>(a);
        else attention_rows_kernel<64, false><<<grid, block, 0, s>>>(a);
    }
    return check_hip(hipGetLastError(), "attention_rows_kernel");
}

}  // namespace qarl
