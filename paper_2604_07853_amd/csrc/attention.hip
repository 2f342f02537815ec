// Attention over the paged cache: the workspace, the launches and the join of the pieces (how a call is split: attention_split.hpp).
#include "attention.hpp"

namespace qarl {

static size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

size_t attention_ws_bytes(int T, int q_heads, int kv_heads, int head_dim, int S, int max_q_len, int max_kv_len)
{
    const AttnPlan p = attention_plan(T, q_heads, kv_heads, S, max_q_len, max_kv_len, 0);
    if (!p.splits) return 0;
    const size_t rows = (size_t)T * q_heads, n = (size_t)p.splits;
    return up256(n * rows * head_dim * 4) + up256(n * rows * 8) + up256(rows * 4);
}

// out = sum over the pieces of 2^(m_i - m) O_i / sum of 2^(m_i - m) l_i, in a fixed order.  A unit of D / 4 lanes holds a row.  A workgroup looks through
// `per` rows, lists those that are in pieces, and joins them: a row of up to kAlone pieces by one unit, a row of more by all of them together.  (A single
// token over 18432 positions: 72 pieces took one unit 26.8 us and take eight 4.0.)
constexpr int kAlone = 8, kJoinRows = 256;

template <int D>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a, AttnParts parts, int per)
{
    constexpr int kLanes = D / 4, kUnits = 256 / kLanes;
    __shared__ f32x4 so[256];
    __shared__ float sm[kUnits], sl[kUnits];
    __shared__ unsigned list[2][kJoinRows];             // rows of few pieces, of many: row - row0, pieces << 16
    __shared__ int listed[2];
    const int unit = threadIdx.x / kLanes, d = threadIdx.x % kLanes * 4;
    const int64_t row0 = (int64_t)blockIdx.x * per;
    if (threadIdx.x < 2) listed[threadIdx.x] = 0;
    __syncthreads();
    if ((int)threadIdx.x < per && row0 + threadIdx.x < parts.rows) {
        const int64_t row = row0 + threadIdx.x;
        const int t = (int)(row / a.q_heads);
        const int n = t >= a.q_offsets[0] && t < a.q_offsets[a.S] ? min(parts.count[row], parts.splits) : 0;    // (none: a row of no sequence)
        if (n > 1) list[n > kAlone][atomicAdd(&listed[n > kAlone], 1)] = threadIdx.x | (unsigned)n << 16;           // (one: written where it was computed)
    }
    __syncthreads();
    float top, sum;
    f32x4 o;
    const auto gather = [&](int64_t row, int n, int from, int step) {
        top = kNegInf;
#pragma unroll 4
        for (int i = from; i < n; i += step) top = fmaxf(top, parts.ml[((int64_t)i * parts.rows + row) * 2]);
        const float tb = top == kNegInf ? 0.f : top;
        sum = 0.f;
        o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int i = from; i < n; i += step) {
            const int64_t at = (int64_t)i * parts.rows + row;
            const float f = __builtin_amdgcn_exp2f(parts.ml[at * 2] - tb);
            sum += f * parts.ml[at * 2 + 1];
            o += *(const f32x4 *)(parts.o + at * D + d) * f;
        }
    };
    const auto finish = [&](int64_t row) {
        store_out4(a, row, D, d, o * inverse_sum(sum));
        if (d == 0 && a.lse) a.lse[row] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
    };
    for (int i = unit; i < listed[0]; i += kUnits) {
        const int64_t row = row0 + (list[0][i] & 0xffff);
        gather(row, (int)(list[0][i] >> 16), 0, 1);
        finish(row);
    }
    for (int i = 0; i < listed[1]; ++i) {
        const int64_t row = row0 + (list[1][i] & 0xffff);
        gather(row, (int)(list[1][i] >> 16), unit, kUnits);
        so[threadIdx.x] = o;
        if (d == 0) {
            sm[unit] = top;
            sl[unit] = sum;
        }
        __syncthreads();
        if (unit == 0) {
            for (int g = 0; g < kUnits; ++g) top = fmaxf(top, sm[g]);
            const float all = top == kNegInf ? 0.f : top;
            sum = 0.f;
            o = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int g = 0; g < kUnits; ++g) {
                const float f = __builtin_amdgcn_exp2f(sm[g] - all);
                sum += f * sl[g];
                o += so[threadIdx.x + g * kLanes] * f;
            }
            finish(row);
        }
        __syncthreads();
    }
}

template <int D>
static int launch_join(const AttnArgs &a, const AttnParts &parts, hipStream_t s)
{
    // rows per workgroup: about as many workgroups as the chip holds at a time
    const int per = (int)max((int64_t)1, min((int64_t)kJoinRows, parts.rows / 2048));
    const int64_t blocks = (parts.rows + per - 1) / per;
    if (blocks > 0x7fffffffLL) {
        set_error("qarl_paged_attention: %lld rows exceed the grid limit", (long long)parts.rows);
        return QARL_ERR_UNSUPPORTED;
    }
    attention_join_kernel<D><<<dim3((unsigned)blocks), dim3(256), 0, s>>>(a, parts, per);
    return check_hip(hipGetLastError(), "attention_join_kernel");
}

int launch_attention(const AttnArgs &a, hipStream_t s)
{
    const int D = a.kv.head_dim;
    AttnPlan p = attention_plan(a.T, a.q_heads, a.kv.kv_heads, a.S, a.max_q_len, a.max_kv_len, a.window);
    AttnParts parts = {};
    parts.rows = (int64_t)a.T * a.q_heads;
    if (p.splits) {
        const size_t n = (size_t)p.splits;
        parts.splits = p.splits;
        parts.o = (float *)a.ws;
        parts.ml = (float *)((char *)a.ws + up256(n * parts.rows * D * 4));
        parts.count = (int32_t *)((char *)parts.ml + up256(n * parts.rows * 8));
    }
    int rc = QARL_OK;
    if (p.tile && (rc = launch_attention_tile(a, p, parts, s))) return rc;
    if (p.few_nr && (rc = launch_attention_few(a, p, parts, s))) return rc;
    if (!p.splits) return QARL_OK;
    return D == 128 ? launch_join<128>(a, parts, s) : launch_join<64>(a, parts, s);
}

}  // namespace qarl
