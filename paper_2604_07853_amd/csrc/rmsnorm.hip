// Residual addition with RMS norm in front of the (quantized) projections, and its backward.
//   forward:  h = x + r (fp32), y = h * rstd * w, rstd = 1 / sqrt(mean h^2 + eps); out: h in the stream's type, y in bf16 and / or
//             as e4m3 codes with a scale per row (the FP quantizer of section 2.2);
//   backward: dx = dh + rstd (g - h rstd^2 mean(g h)), g = dy w;  dw = sum over rows of dy h rstd.
// Both are bound by memory (about ten operations per element): every element is requested once, with 16-byte loads, and a row
// stays in registers between its reductions and its outputs.
#include "common.hpp"

namespace qarl {

constexpr int kNormThreads = 256;

// Eight stream elements: fp32 [8] or bf16 [8]
template <bool F32>
__device__ __forceinline__ void load_stream8(const void *base, int64_t at, float (&t)[8])
{
    if (F32) {
        const f32x4 *p = (const f32x4 *)((const float *)base + at);
        const f32x4 a = p[0], b = p[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            t[i] = a[i];
            t[4 + i] = b[i];
        }
    } else {
        bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)base + at), t);
    }
}

template <bool F32>
__device__ __forceinline__ void store_stream8(void *base, int64_t at, const float (&t)[8])
{
    if (F32) {
        f32x4 *p = (f32x4 *)((float *)base + at);
        p[0] = f32x4{t[0], t[1], t[2], t[3]};
        p[1] = f32x4{t[4], t[5], t[6], t[7]};
    } else {
        *(u32x4 *)((uint16_t *)base + at) = f32_to_bf16x8(t);
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
template <int kLanes, int kChunks, bool F32>
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
            bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.x + row * a.x_stride + i * 8), h[c]);
            if (a.res) {
                float r[8];
                load_stream8<F32>(a.res, row * a.res_stride + i * 8, r);
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
        if (a.res_out) store_stream8<F32>(a.res_out, row * a.res_out_stride + i * 8, h[c]);
        float w[8];
        bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.w + i * 8), w);
#pragma unroll
        for (int e = 0; e < 8; ++e) h[c][e] = h[c][e] * rstd * w[e];
        if (a.y) *(u32x4 *)((uint16_t *)a.y + row * a.y_stride + i * 8) = f32_to_bf16x8(h[c]);
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
        if (live && i < n8) *(u32x2 *)((uint8_t *)a.codes + row * a.K + i * 8) = sc.quantize8(h[c]);
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
    if (a.stream_f32) rmsnorm_kernel<kLanes, kChunks, true><<<dim3((unsigned)blocks), dim3(kNormThreads), 0, s>>>(a);
    else rmsnorm_kernel<kLanes, kChunks, false><<<dim3((unsigned)blocks), dim3(kNormThreads), 0, s>>>(a);
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
// A workgroup takes rows blockIdx.x, blockIdx.x + gridDim.x, ... (kLanes == 64: four at a time, one per wavefront); a lane owns
// the same columns in every row and keeps their dw sums in registers.  Partial sums go to [gridDim.x][K], in a fixed order.
template <int kLanes, int kChunks, bool F32>
__global__ __launch_bounds__(kNormThreads) void rmsnorm_backward_kernel(NormGradArgs a)
{
    constexpr int kRows = kNormThreads / kLanes;
    __shared__ float part[4][4];
    __shared__ float fold[kRows > 1 ? kChunks * kLanes * 8 : 1];
    const int lane = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;
    const int n8 = a.K / 8;
    float dw[kChunks][8];
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[c][e] = 0.f;
    int turn = 0;     // the workgroup reductions of neighbouring rows use different slots
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.rows; row0 += (int64_t)gridDim.x * kRows, turn ^= 2) {
        const int64_t row = row0 + sub;
        const bool live = row < a.rows;
        float h[kChunks][8], g[kChunks][8];
        float sq = 0.f, gh = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int i = lane + c * kLanes;
#pragma unroll
            for (int e = 0; e < 8; ++e) h[c][e] = g[c][e] = 0.f;
            if (live && i < n8) {
                load_stream8<F32>(a.h, row * a.h_stride + i * 8, h[c]);
                bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.dy + row * a.dy_stride + i * 8), g[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int i = lane + c * kLanes;
            float w[8];
            bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.w + (i < n8 ? i : 0) * 8), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sq = fmaf(h[c][e], h[c][e], sq);
                gh = fmaf(g[c][e] * w[e], h[c][e], gh);
            }
        }
        sq = row_reduce<kLanes, false>(sq, part, turn);
        gh = row_reduce<kLanes, false>(gh, part, turn + 1);
        const float rstd = 1.0f / sqrtf(sq / (float)a.K + a.eps);
        const float k = rstd * rstd * (gh / (float)a.K);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            const int i = lane + c * kLanes;
            if (!live || i >= n8) continue;
            float w[8], d[8];
            bf16x8_to_f32(*(const u32x4 *)((const uint16_t *)a.w + i * 8), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = 0.f;
            if (a.dh) load_stream8<F32>(a.dh, row * a.dh_stride + i * 8, d);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                dw[c][e] = fmaf(g[c][e] * rstd, h[c][e], dw[c][e]);
                d[e] += rstd * fmaf(-h[c][e], k, g[c][e] * w[e]);
            }
            store_stream8<F32>(a.dx, row * a.dx_stride + i * 8, d);
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
                        float *f = &fold[(c * kLanes + lane) * 8 + e];
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
        if (i < n8) store_stream8<true>(a.partials, (int64_t)blockIdx.x * a.K + i * 8, dw[c]);
    }
}

// dw[k] = sum over the workgroups' partials: 32 columns per workgroup, 32 threads per column, then a tree in LDS.
__global__ __launch_bounds__(1024) void rmsnorm_dw_kernel(const float *__restrict__ partials, int64_t groups, int K, void *dw, int dw_f32)
{
    __shared__ float part[32][33];
    const int col = threadIdx.x & 31, lane = threadIdx.x >> 5, k = blockIdx.x * 32 + col;
    float v = 0.f;
    if (k < K)
        for (int64_t g = lane; g < groups; g += 32) v += partials[g * K + k];
    part[lane][col] = v;
    __syncthreads();
    for (int o = 16; o > 0; o >>= 1) {
        if (lane < o) part[lane][col] += part[lane + o][col];
        __syncthreads();
    }
    if (lane == 0 && k < K) {
        if (dw_f32) ((float *)dw)[k] = part[0][col];
        else ((uint16_t *)dw)[k] = f32_to_bf16_hw(part[0][col]);
    }
}

int64_t rmsnorm_backward_groups(int64_t rows, int K)
{
    const int per = K <= 4096 ? 4 : 1;
    const int64_t g = (rows + per - 1) / per;
    return g < 512 ? g : 512;
}

template <int kLanes, int kChunks>
static int launch_norm_grad_as(const NormGradArgs &a, hipStream_t s)
{
    const unsigned groups = (unsigned)rmsnorm_backward_groups(a.rows, a.K);
    if (a.stream_f32) rmsnorm_backward_kernel<kLanes, kChunks, true><<<dim3(groups), dim3(kNormThreads), 0, s>>>(a);
    else rmsnorm_backward_kernel<kLanes, kChunks, false><<<dim3(groups), dim3(kNormThreads), 0, s>>>(a);
    return check_hip(hipGetLastError(), "rmsnorm_backward_kernel");
}

int launch_rmsnorm_backward(const NormGradArgs &a, hipStream_t s)
{
    const int64_t groups = rmsnorm_backward_groups(a.rows, a.K);
    int rc = QARL_OK;
    if (groups > 0) {
        if (a.K <= 512) rc = launch_norm_grad_as<64, 1>(a, s);
        else if (a.K <= 2048) rc = launch_norm_grad_as<64, 4>(a, s);
        else if (a.K <= 4096) rc = launch_norm_grad_as<64, 8>(a, s);
        else if (a.K <= 8192) rc = launch_norm_grad_as<256, 4>(a, s);
        else rc = launch_norm_grad_as<256, 8>(a, s);
    }
    if (rc || !a.dw) return rc;
    rmsnorm_dw_kernel<<<dim3((unsigned)((a.K + 31) / 32)), dim3(1024), 0, s>>>(a.partials, groups, a.K, a.dw, a.dw_f32);
    return check_hip(hipGetLastError(), "rmsnorm_dw_kernel");
}

}  // namespace qarl
