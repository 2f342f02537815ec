// The paged KV cache: writing new tokens (quantized on the way, or copied) and reading sequences back in bf16.
// Layout [page][head][offset][head_dim]: the tokens of a page and head lie behind one another, which is what attention streams.
// Both kernels are bound by memory; a thread moves eight elements of k and the same eight of v.  Writing 16384 tokens of 4 x 128 in bf16 (67 MB, which the
// last-level cache holds) takes 11.4 us, 5.9 TB/s; 256 tokens in e4m3 4.1 us, which is the launch.
// e2m1: a scale for each quarter of a row, 2^e with the smallest e for which the quarter's largest size is at most 6 2^e: the matrix and conversion instructions
// take such a byte as it is, and codes times scale are exact in bf16.
#include "common.hpp"

namespace qarl {

constexpr int kKvThreads = 256;

// Maximum over the D / 8 lanes that own a row of the cache
template <int D>
__device__ __forceinline__ float head_max(float v)
{
#pragma unroll
    for (int o = D / 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

template <int D, int FMT>
__global__ __launch_bounds__(kKvThreads) void kv_write_kernel(KvArgs c, const uint16_t *__restrict__ k, int64_t kts, int64_t khs,
                                                              const uint16_t *__restrict__ v, int64_t vts, int64_t vhs, int64_t T,
                                                              const int64_t *__restrict__ slots)
{
    constexpr int kChunks = D / 8;
    const int64_t i = (int64_t)blockIdx.x * kKvThreads + threadIdx.x;
    const int chunk = (int)(i % kChunks);
    const int64_t th = i / kChunks, t = th / c.kv_heads;
    const int h = (int)(th - t * c.kv_heads);
    const int64_t slot = t < T ? slots[t] : -1;
    const bool live = slot >= 0 && slot < ((int64_t)c.num_pages << c.page_shift);   // the lanes of a row agree
    u32x4 kv[2] = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
    if (live) {
        kv[0] = *(const u32x4 *)(k + t * kts + h * khs + chunk * 8);
        kv[1] = *(const u32x4 *)(v + t * vts + h * vhs + chunk * 8);
    }
    const int64_t page = slot >> c.page_shift;
    const int64_t to = ((page * c.kv_heads + h) << c.page_shift) + (slot & ((1 << c.page_shift) - 1));   // row of the cache
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        if (FMT == QARL_KV_E4M3) {
            float f[8];
            bf16x8_to_f32(kv[w], f);
            const LaneScale sc(head_max<D>(LaneScale::absmax8(f, 0.f)));
            if (!live) continue;
            *(u32x2 *)((uint8_t *)(w ? c.v : c.k) + to * D + chunk * 8) = sc.quantize8(f);
            if (chunk == 0) (w ? c.v_scales : c.k_scales)[to] = sc.stored();
        } else if (FMT == QARL_KV_E2M1) {
            constexpr int kGroupLanes = kChunks / 4;        // lanes of a group of D / 4 elements
            float f[8];
            bf16x8_to_f32(kv[w], f);
            float absmax = LaneScale::absmax8(f, 0.f);
#pragma unroll
            for (int o = kGroupLanes / 2; o > 0; o >>= 1) absmax = fmaxf(absmax, __shfl_xor(absmax, o, 64));
            const E2m1Scale sc(absmax);
            if (!live) continue;
            *(uint32_t *)((uint8_t *)(w ? c.v : c.k) + to * (D / 2) + chunk * 4) = sc.quantize8(f);
            if (chunk % kGroupLanes == 0) ((uint8_t *)(w ? c.v_scales : c.k_scales))[to * 4 + chunk / kGroupLanes] = sc.byte;
        } else if (live) {
            *(u32x4 *)((uint16_t *)(w ? c.v : c.k) + to * D + chunk * 8) = kv[w];
        }
    }
}

int launch_kv_write(const KvArgs &c, const void *k, int64_t kts, int64_t khs, const void *v, int64_t vts, int64_t vhs, int64_t T,
                    const int64_t *slots, hipStream_t s)
{
    const int64_t blocks = (T * c.kv_heads * (c.head_dim / 8) + kKvThreads - 1) / kKvThreads;
    if (blocks > 0x7fffffffLL) {
        set_error("qarl_kv_cache_write: %lld tokens exceed the grid limit", (long long)T);
        return QARL_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)blocks), block(kKvThreads);
    const uint16_t *kp = (const uint16_t *)k, *vp = (const uint16_t *)v;
#define QARL_KV_WRITE(D) \
    if (c.fmt == QARL_KV_E4M3) kv_write_kernel<D, QARL_KV_E4M3><<<grid, block, 0, s>>>(c, kp, kts, khs, vp, vts, vhs, T, slots); \
    else if (c.fmt == QARL_KV_E2M1) kv_write_kernel<D, QARL_KV_E2M1><<<grid, block, 0, s>>>(c, kp, kts, khs, vp, vts, vhs, T, slots); \
    else kv_write_kernel<D, QARL_KV_BF16><<<grid, block, 0, s>>>(c, kp, kts, khs, vp, vts, vhs, T, slots)
    if (c.head_dim == 128) {
        QARL_KV_WRITE(128);
    } else {
        QARL_KV_WRITE(64);
    }
#undef QARL_KV_WRITE
    return check_hip(hipGetLastError(), "kv_write_kernel");
}

// A workgroup takes kReadRows output rows.  Its first threads look their rows' sequences up (the last s with offsets[s] <= row) and
// leave the page's first cache row in LDS; then all threads copy.
// 8 x 18432 positions of e4m3, 458 MB: 93.8 us with 32 rows and cached accesses, 86.3 with 16 and accesses that bypass the caches (5.3 TB/s); 37 short
// sequences, 39 MB: 9.5 us cached, 10.4 past the caches: those are for calls that would not stay in them.  Calls of few rows take four a workgroup: more of them
// wait for lengths and pages at once (37 sequences of 15 positions in e4m3 4.7 -> 3.7 us, of 150 in bf16 5.6 -> 5.5, of 260 7.3 -> 8.5; where four rows of all heads leave threads without work, as two heads of 128 do,
// up to fewer rows: 37 of 50 in bf16 3.7 -> 3.5, 64 of 60 3.9 -> 4.0, 65 of 90 4.4 -> 4.75).  Many sequences' search begins
// among some of the offsets in LDS (300 of 30 in bf16 8.0 -> 7.1, 128 of 200 of two heads 10.9 -> 10.2; 37 of 15 4.0 -> 4.2, 65 of 60 of two heads 4.0 -> 4.15).
constexpr int kReadFew = 6144, kReadFewNarrow = 2560, kReadDirect = 96;
constexpr int64_t kReadCached = (int64_t)64 << 20;

template <int D, int FMT, bool NT, int kReadRows>
__global__ __launch_bounds__(kKvThreads) void kv_read_kernel(KvArgs c, const int32_t *__restrict__ table, int64_t table_stride, int table_width,
                                                             const int32_t *__restrict__ offsets, int S, int64_t total,
                                                             uint16_t *__restrict__ k_out, uint16_t *__restrict__ v_out)
{
    constexpr int kChunks = D / 8;
    __shared__ int64_t from[kReadRows];     // cache row of head 0, or -1
    __shared__ int32_t every[kKvThreads + 1];           // the offset of every `step`-th sequence, and the end
    const int64_t row0 = (int64_t)blockIdx.x * kReadRows;
    const int step = (S + kKvThreads - 1) / kKvThreads;
    const bool many = S > kReadDirect;
    if (many) {
        for (int i = threadIdx.x; i <= kKvThreads; i += kKvThreads) every[i] = offsets[min((int64_t)i * step, (int64_t)S)];
        __syncthreads();
    }
    if (threadIdx.x < kReadRows) {
        const int64_t row = row0 + threadIdx.x;
        int64_t at = -1;
        if (row < total && S > 0 && row >= offsets[0] && row < offsets[S]) {
            int lo = 0, hi = S;
            if (many) {
                hi = kKvThreads;            // every[lo] <= row < every[hi]
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (every[mid] <= row) lo = mid;
                    else hi = mid;
                }
                hi = min(hi * step, S);     // offsets[lo] <= row < offsets[hi]
                lo *= step;
            }
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (offsets[mid] <= row) lo = mid;
                else hi = mid;
            }
            const int64_t pos = row - offsets[lo], col = pos >> c.page_shift;
            if (col < table_width) {
                const int page = table[lo * table_stride + col];
                if (page >= 0 && page < c.num_pages)
                    at = (((int64_t)page * c.kv_heads) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
            }
        }
        from[threadIdx.x] = at;
    }
    __syncthreads();
    const int per_row = c.kv_heads * kChunks;
    const int rows = (int)(total - row0 < kReadRows ? total - row0 : kReadRows);
    for (int i = threadIdx.x; i < rows * per_row; i += kKvThreads) {
        const int r = i / per_row, j = i - r * per_row, h = j / kChunks, chunk = j % kChunks;
        const int64_t at = from[r];
        u32x4 kv[2] = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
        if (at >= 0) {
            const int64_t src = at + ((int64_t)h << c.page_shift);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                if (FMT == QARL_KV_E2M1) {
                    const uint32_t q4 = load_as<NT, uint32_t>((const uint8_t *)(w ? c.v : c.k) + src * (D / 2) + chunk * 4);
                    kv[w] = widen_e2m1x8(q4, e2m1_scale((w ? c.v_bytes() : c.k_bytes())[src * 4 + chunk / (kChunks / 4)]));
                } else if (FMT == QARL_KV_E4M3) {
                    const u32x2 q8 = load_as<NT, u32x2>((const uint8_t *)(w ? c.v : c.k) + src * D + chunk * 8);
                    const float sc = (w ? c.v_scales : c.k_scales)[src];
                    float f[8];
                    bf16x8_to_f32(e4m3_as_bf16x8(q8), f);
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] *= sc;
                    kv[w] = f32_to_bf16x8(f);
                } else {
                    kv[w] = load_as<NT, u32x4>((const uint16_t *)(w ? c.v : c.k) + src * D + chunk * 8);
                }
            }
        }
        const int64_t o = ((row0 + r) * c.kv_heads + h) * D + chunk * 8;
        store_as<NT>(k_out + o, kv[0]);
        store_as<NT>(v_out + o, kv[1]);
    }
}

int launch_kv_read(const KvArgs &c, const int32_t *table, int64_t table_stride, int table_width, const int32_t *offsets, int S,
                   int64_t total, void *k_out, void *v_out, hipStream_t s)
{
    const bool nt = total * c.kv_heads * c.head_dim * (c.fmt == QARL_KV_BF16 ? 8 : c.fmt == QARL_KV_E4M3 ? 6 : 5) > kReadCached;
    const int rows = total <= (4 * c.kv_heads * (c.head_dim / 8) >= kKvThreads ? kReadFew : kReadFewNarrow) && !nt ? 4 : 16;
    const int64_t blocks = (total + rows - 1) / rows;
    if (blocks > 0x7fffffffLL) {
        set_error("qarl_kv_cache_read: %lld rows exceed the grid limit", (long long)total);
        return QARL_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)blocks), block(kKvThreads);
    uint16_t *ko = (uint16_t *)k_out, *vo = (uint16_t *)v_out;
#define QARL_KV_READ(D, FMT, NT, ROWS) kv_read_kernel<D, FMT, NT, ROWS><<<grid, block, 0, s>>>(c, table, table_stride, table_width, offsets, S, total, ko, vo)
#define QARL_KV_READ_AS(D, FMT) \
    if (rows == 4) QARL_KV_READ(D, FMT, false, 4); \
    else if (nt) QARL_KV_READ(D, FMT, true, 16); \
    else QARL_KV_READ(D, FMT, false, 16)
#define QARL_KV_READ_FROM(D) \
    if (c.fmt == QARL_KV_E4M3) { \
        QARL_KV_READ_AS(D, QARL_KV_E4M3); \
    } else if (c.fmt == QARL_KV_E2M1) { \
        QARL_KV_READ_AS(D, QARL_KV_E2M1); \
    } else { \
        QARL_KV_READ_AS(D, QARL_KV_BF16); \
    }
    if (c.head_dim == 128) {
        QARL_KV_READ_FROM(128)
    } else {
        QARL_KV_READ_FROM(64)
    }
#undef QARL_KV_READ_FROM
#undef QARL_KV_READ_AS
#undef QARL_KV_READ
    return check_hip(hipGetLastError(), "kv_read_kernel");
}

}  // namespace qarl
