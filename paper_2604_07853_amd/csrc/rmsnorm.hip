// Residual addition with RMS norm in front of the (quantized) projections, and its backward.
//   forward:  h = x + r (fp32), y = h * rstd * w, rstd = 1 / sqrt(mean h^2 + eps); out: h in the stream's type, y in bf16 and / or
//             as e4m3 codes with a scale per row (the FP quantizer of section 2.2);
//   backward: dx = dh + rstd (g - h rstd^2 mean(g h)), g = dy w;  dw = sum over rows of dy h rstd.
// Both are bound by memory (about ten operations per element): every element is requested once, with 16-byte loads, and a row
// stays in registers between its reductions and its outputs.  Forward of one row of 2048: 3.7 us, the launch; 16384 rows with e4m3 output: 42 us,
// 235 MB, 5.6 TB/s.  Backward of the same rows: 47 us, 273 MB, 5.8 TB/s, and 5 us for the sums of dw.
#include "common.hpp"

namespace qarl {

constexpr int kNormThreads = 256;

// Calls that move more than this bypass the caches (a quarter of the last one): nothing of them would still be there for the next kernel.  Norm of
// 16384 x 2048 with e4m3 output 55.3 -> 45.1 us (5.2 TB/s), 4000 x 8192 fp32 88.0 -> 79.2; 256 x 2048 loses by it, 7.2 -> 8.1.
constexpr int64_t kNormCached = (int64_t)64 << 20;

// Eight stream elements as they lie in memory: fp32 [8] or bf16 [8]
template <bool F32>
struct Raw8 {
    u32x4 w[F32 ? 2 : 1];
    template <bool NT>
    __device__ __forceinline__ void load(const void *base, int64_t at)
    {
        const char *p = (const char *)base + at * (F32 ? 4 : 2);
        w[0] = load_as<NT, u32x4>(p);
        if constexpr (F32) w[1] = load_as<NT, u32x4>(p + 16);
    }
    __device__ __forceinline__ void widen(float (&t)[8]) const
    {
        if constexpr (F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = __uint_as_float(w[i >> 2][i & 3]);
        } else {
            bf16x8_to_f32(w[0], t);
        }
    }
};

template <bool F32, bool NT>
__device__ __forceinline__ void store_stream8(void *base, int64_t at, const float (&t)[8])
{
    if constexpr (F32) {
        float *p = (float *)base + at;
        store_as<NT>(p, f32x4{t[0], t[1], t[2], t[3]});
        store_as<NT>(p + 4, f32x4{t[4], t[5], t[6], t[7]});
    } else {
        store_as<NT>((uint16_t *)base + at, f32_to_bf16x8(t));
    }
}

// Sum / maximum over the kLanes lanes that own a row: lanes of a wavefront, or (kLanes == 256) the whole workgroup by way of
// `part`; `slot` gives every reduction of a row its own four floats, so that one barrier each is enough.
template <int kLanes, bool MAX>
__device__ __forceinline__ float row_reduce(float v, float (*part)[4], int slot)
{
    constexpr int kIn = kLanes < 64 ? kLanes : 64;
#pragma unroll
    for (int o = kIn / 2; o > 0; o >>= 1) {
        const float u = __shfl_xor(v, o, 64);
        v = MAX ? fmaxf(v, u) : v + u;
    }
    if (kLanes == kNormThreads) {
        if ((threadIdx.x & 63) == 0) part[slot][threadIdx.x >> 6] = v;
        __syncthreads();
        v = MAX ? fmaxf(fmaxf(part[slot][0], part[slot][1]), fmaxf(part[slot][2], part[slot][3]))
                : (part[slot][0] + part[slot][1]) + (part[slot][2] + part[slot][3]);
    }
    return v;
}

// kLanes lanes per row (16: four rows per wavefront, 64, or 256: a workgroup), kChunks times eight elements per lane.
template <int kLanes, int kChunks, bool F32, bool NT>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_kernel(NormArgs a)
{
    __shared__ float part[2][4];
    const int lane = threadIdx.x % kLanes;
    const int64_t row = (int64_t)blockIdx.x * (kNormThreads / kLanes) + threadIdx.x / kLanes;
    const int n8 = a.K / 8;
    const bool live = row < a.rows;     // lanes of other rows of the wavefront take part in its shuffles
    float h[kChunks][8];
    float sq = 0.f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int i = lane + c * kLanes;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] = 0.f;
        if (live && i < n8) {
            bf16x8_to_f32(load_as<NT, u32x4>((const uint16_t *)a.x + row * a.x_stride + i * 8), h[c]);
            if (a.res) {
                Raw8<F32> raw;
                float r[8];
                raw.template load<NT>(a.res, row * a.res_stride + i * 8);
                raw.widen(r);
#pragma unroll
                for (int e = 0; e < 8; ++e) h[c][e] += r[e];
            }
        }
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = fmaf(h[c][e], h[c][e], sq);
    sq = row_reduce<kLanes, false>(sq, part, 0);
    const float rstd = 1.0f / sqrtf(sq / (float)a.K + a.eps);
    float am = 0.f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int i = lane + c * kLanes;
        if (!live || i >= n8) continue;
        if (a.res_out) store_stream8<F32, NT>(a.res_out, row * a.res_out_stride + i * 8, h[c]);
        float w[8];
        bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.w + i * 8), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] = h[c][e] * rstd * w[e];
        if (a.y) store_as<NT>((uint16_t *)a.y + row * a.y_stride + i * 8, f32_to_bf16x8(h[c]));
        if (a.codes) {
            if (a.via_bf16) bf16x8_to_f32(f32_to_bf16x8(h[c]), h[c]);
            am = LaneScale::absmax8(h[c], am);
        }
    }
    if (!a.codes) return;
    am = row_reduce<kLanes, true>(am, part, 1);
    const LaneScale sc(am);
    if (live && lane == 0) a.scales[row] = sc.stored();
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int i = lane + c * kLanes;
        if (live && i < n8) store_as<NT>((uint8_t *)a.codes + row * a.K + i * 8, sc.quantize8(h[c]));
    }
}

template <int kLanes, int kChunks>
static int launch_norm_as(const NormArgs &a, hipStream_t s)
{
    constexpr int kRows = kNormThreads / kLanes;
    const int64_t blocks = (a.rows + kRows - 1) / kRows;
    if (blocks > 0x7fffffffLL) {
        set_error("qarl_add_rmsnorm: %lld rows exceed the grid limit", (long long)a.rows);
        return QARL_ERR_UNSUPPORTED;
    }
    const int st = a.stream_f32 ? 4 : 2;
    const bool nt = a.rows * a.K * (2 + (a.res ? st : 0) + (a.res_out ? st : 0) + (a.y ? 2 : 0) + (a.codes ? 1 : 0)) > kNormCached;
    const dim3 grid((unsigned)blocks), block(kNormThreads);
    if (a.stream_f32) {
        if (nt) rmsnorm_kernel<kLanes, kChunks, true, true><<<grid, block, 0, s>>>(a);
        else rmsnorm_kernel<kLanes, kChunks, true, false><<<grid, block, 0, s>>>(a);
    } else {
        if (nt) rmsnorm_kernel<kLanes, kChunks, false, true><<<grid, block, 0, s>>>(a);
        else rmsnorm_kernel<kLanes, kChunks, false, false><<<grid, block, 0, s>>>(a);
    }
    return check_hip(hipGetLastError(), "rmsnorm_kernel");
}

int launch_rmsnorm(const NormArgs &a, hipStream_t s)
{
    if (a.K <= 128) return launch_norm_as<16, 1>(a, s);
    if (a.K <= 512) return launch_norm_as<16, 4>(a, s);
    if (a.K <= 2048) return launch_norm_as<64, 4>(a, s);
    if (a.K <= 4096) return launch_norm_as<256, 2>(a, s);
    if (a.K <= 8192) return launch_norm_as<256, 4>(a, s);
    return launch_norm_as<256, 8>(a, s);
}

// ------------------------------------------------------------ backward --
// A workgroup takes rows blockIdx.x, blockIdx.x + gridDim.x, ... (kLanes == 64: four at a time, one per wavefront); a lane owns the same columns in
// every row and keeps their dw sums in registers.  The next row is requested before the current one is worked on: with a row at a time the loads of
// dh waited for both reductions.  Partial sums of dw go to [gridDim.x][K], in a fixed order.
template <int kLanes, int kChunks, bool F32>
__global__ __launch_bounds__(kLanes > kNormThreads ? kLanes : kNormThreads) void rmsnorm_backward_kernel(NormGradArgs a)
{
    constexpr int kThreads = kLanes > kNormThreads ? kLanes : kNormThreads, kRows = kThreads / kLanes, kWaves = kLanes / 64;
    __shared__ float part[2][2][kWaves];
    __shared__ float fold[kRows > 1 ? kChunks * kLanes * 8 : 1];
    const int lane = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;
    const int n8 = a.K / 8;
    float dw[kChunks][8];
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[c][e] = 0.f;
    struct Row {
        Raw8<F32> h[kChunks], dh[kChunks];
        Raw8<false> dy[kChunks];
    };
    auto request = [&](int64_t row, Row &r) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int i = lane + c * kLanes;
            r.h[c] = r.dh[c] = Raw8<F32>{};
            r.dy[c] = Raw8<false>{};
            if (row >= a.rows || i >= n8) continue;
            r.h[c].template load<false>(a.h, row * a.h_stride + i * 8);
            r.dy[c].template load<false>(a.dy, row * a.dy_stride + i * 8);
            if (a.dh) r.dh[c].template load<false>(a.dh, row * a.dh_stride + i * 8);
        }
    };
    Row next;
    request((int64_t)blockIdx.x * kRows + sub, next);
    int turn = 0;     // neighbouring rows meet in different places of `part`
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.rows; row0 += (int64_t)gridDim.x * kRows, turn ^= 1) {
        const int64_t row = row0 + sub;
        const Row now = next;
        request(row + (int64_t)gridDim.x * kRows, next);
        float sq = 0.f, gh = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int i = lane + c * kLanes;
            float h[8], g[8], w[8];
            now.h[c].widen(h);
            now.dy[c].widen(g);
            bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.w + (i < n8 ? i : 0) * 8), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sq = fmaf(h[e], h[e], sq);
                gh = fmaf(g[e] * w[e], h[e], gh);
            }
        }
        sq = wave_sum(sq);
        gh = wave_sum(gh);
        if (kWaves > 1) {
            if ((threadIdx.x & 63) == 0) {
                part[turn][0][threadIdx.x >> 6] = sq;
                part[turn][1][threadIdx.x >> 6] = gh;
            }
            lds_barrier();
            sq = gh = 0.f;
#pragma unroll
            for (int v = 0; v < kWaves; ++v) {
                sq += part[turn][0][v];
                gh += part[turn][1][v];
            }
        }
        const float rstd = 1.0f / sqrtf(sq / (float)a.K + a.eps);
        const float k = rstd * rstd * (gh / (float)a.K);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int i = lane + c * kLanes;
            if (row >= a.rows || i >= n8) continue;
            float h[8], g[8], w[8], d[8];
            now.h[c].widen(h);
            now.dy[c].widen(g);
            now.dh[c].widen(d);
            bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.w + i * 8), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[c][e] = fmaf(g[e] * rstd, h[e], dw[c][e]);
                d[e] += rstd * fmaf(-h[e], k, g[e] * w[e]);
            }
            store_stream8<F32, false>(a.dx, row * a.dx_stride + i * 8, d);
        }
    }
    if (!a.dw) return;
    if (kRows > 1) {    // the wavefronts' sums, one after the other
        for (int w = 0; w < kRows; ++w) {
            if (sub == w) {
#pragma unroll
                for (int c = 0; c < kChunks; ++c)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float *f = &fold[(c * 8 + e) * kLanes + lane];
                        dw[c][e] += w > 0 ? *f : 0.f;
                        *f = dw[c][e];
                    }
            }
            __syncthreads();
        }
        if (sub != kRows - 1) return;
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        const int i = lane + c * kLanes;
        if (i < n8) store_stream8<true, false>(a.partials, (int64_t)blockIdx.x * a.K + i * 8, dw[c]);
    }
}

// dw[k] = sum over the workgroups' partials: 32 columns per workgroup, 128 threads per four of them, then a tree in LDS.
__global__ __launch_bounds__(1024) void rmsnorm_dw_kernel(const float *__restrict__ partials, int groups, int K, void *dw, int dw_f32)
{
    __shared__ f32x4 part[128][9];
    const int col = threadIdx.x & 7, lane = threadIdx.x >> 3, k = blockIdx.x * 32 + col * 4;
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (k < K) {
#pragma unroll 4
        for (int g = lane; g < groups; g += 128) v += *(const f32x4 *)(partials + (int64_t)g * K + k);
    }
    part[lane][col] = v;
    __syncthreads();
    for (int o = 64; o > 0; o >>= 1) {
        if (lane < o) part[lane][col] += part[lane + o][col];
        __syncthreads();
    }
    if (lane == 0 && k < K) {
        const f32x4 t = part[0][col];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (dw_f32) ((float *)dw)[k + e] = t[e];
            else ((uint16_t *)dw)[k + e] = f32_to_bf16_hw(t[e]);
        }
    }
}

// Workgroups: more keep more rows in flight, and leave more partial sums behind.  Measured with 256 / 512 / 768 / 1024 (us): 16384 x 2048 bf16
// 67.6 / 58.2 / 66.9 / 62.9 (768 leave an uneven last round), 8192 x 4096 76.6 / 61.6 / 56.0 / 57.7, 1733 x 4096 fp32 25.9 / 24.0 / 24.8 / 28.2,
// 2000 x 16384 (512 threads) 64.3 / 71.6 / 78.8 / 88.0.
int64_t rmsnorm_backward_groups(int64_t rows, int K)
{
    const int per = K <= 2048 ? 4 : 1;
    const int64_t g = (rows + per - 1) / per, most = K <= 2048 ? 512 : K <= 4096 ? 768 : K <= 8192 ? 512 : 256;
    return g < most ? g : most;
}

template <int kLanes, int kChunks>
static int launch_norm_grad_as(const NormGradArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)rmsnorm_backward_groups(a.rows, a.K)), block(kLanes > kNormThreads ? kLanes : kNormThreads);
    if (a.stream_f32) rmsnorm_backward_kernel<kLanes, kChunks, true><<<grid, block, 0, s>>>(a);
    else rmsnorm_backward_kernel<kLanes, kChunks, false><<<grid, block, 0, s>>>(a);
    return check_hip(hipGetLastError(), "rmsnorm_backward_kernel");
}

int launch_rmsnorm_backward(const NormGradArgs &a, hipStream_t s)
{
    const int64_t groups = rmsnorm_backward_groups(a.rows, a.K);
    int rc = QARL_OK;
    if (groups > 0) {
        if (a.K <= 512) rc = launch_norm_grad_as<64, 1>(a, s);
        else if (a.K <= 2048) rc = launch_norm_grad_as<64, 4>(a, s);
        else if (a.K <= 4096) rc = launch_norm_grad_as<256, 2>(a, s);
        else if (a.K <= 8192) rc = launch_norm_grad_as<256, 4>(a, s);
        else rc = launch_norm_grad_as<512, 4>(a, s);
    }
    if (rc || !a.dw) return rc;
    rmsnorm_dw_kernel<<<dim3((unsigned)((a.K + 31) / 32)), dim3(1024), 0, s>>>(a.partials, (int)groups, a.K, a.dw, a.dw_f32);
    return check_hip(hipGetLastError(), "rmsnorm_dw_kernel");
}

}  // namespace qarl
