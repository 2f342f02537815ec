// The paged KV cache: writing new tokens (quantized on the way, or copied) and reading sequences back in bf16.
// Layout [page][head][offset][head_dim]: the tokens of a page and head lie behind one another, which is what attention streams.
// Both kernels are bound by memory; a thread moves eight elements of k and the same eight of v.  Writing 16384 tokens of 4 x 128 in bf16 (67 MB, which the
// last-level cache holds) takes 11.4 us, 5.9 TB/s; 256 tokens in e4m3 4.1 us, which is the launch.
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

template <int D, bool E4M3>
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
        if (E4M3) {
            float f[8];
            bf16x8_to_f32(kv[w], f);
            const LaneScale sc(head_max<D>(LaneScale::absmax8(f, 0.f)));
            if (!live) continue;
            *(u32x2 *)((uint8_t *)(w ? c.v : c.k) + to * D + chunk * 8) = sc.quantize8(f);
            if (chunk == 0) (w ? c.v_scales : c.k_scales)[to] = sc.stored();
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
    const bool e4m3 = c.fmt == QARL_KV_E4M3;
    if (c.head_dim == 128) {
        if (e4m3) kv_write_kernel<128, true><<<grid, block, 0, s>>>(c, kp, kts, khs, vp, vts, vhs, T, slots);
        else kv_write_kernel<128, false><<<grid, block, 0, s>>>(c, kp, kts, khs, vp, vts, vhs, T, slots);
    } else {
        if (e4m3) kv_write_kernel<64, true><<<grid, block, 0, s>>>(c, kp, kts, khs, vp, vts, vhs, T, slots);
        else kv_write_kernel<64, false><<<grid, block, 0, s>>>(c, kp, kts, khs, vp, vts, vhs, T, slots);
    }
    return check_hip(hipGetLastError(), "kv_write_kernel");
}

// A workgroup takes kReadRows output rows.  Its first threads look their rows' sequences up (the last s with offsets[s] <= row) and
// leave the page's first cache row in LDS; then all threads copy.
// 8 x 18432 positions of e4m3, 458 MB: 93.8 us with 32 rows and cached accesses, 86.3 with 16 and accesses that bypass the caches (5.3 TB/s); 37 short
// sequences, 39 MB: 9.5 us cached, 10.4 past the caches: those are for calls that would not stay in them.
constexpr int kReadRows = 16;
constexpr int64_t kReadCached = (int64_t)64 << 20;

template <int D, bool E4M3, bool NT>
__global__ __launch_bounds__(kKvThreads) void kv_read_kernel(KvArgs c, const int32_t *__restrict__ table, int64_t table_stride, int table_width,
                                                             const int32_t *__restrict__ offsets, int S, int64_t total,
                                                             uint16_t *__restrict__ k_out, uint16_t *__restrict__ v_out)
{
    constexpr int kChunks = D / 8;
    __shared__ int64_t from[kReadRows];     // cache row of head 0, or -1
    const int64_t row0 = (int64_t)blockIdx.x * kReadRows;
    if (threadIdx.x < kReadRows) {
        const int64_t row = row0 + threadIdx.x;
        int64_t at = -1;
        if (row < total && S > 0 && row >= offsets[0] && row < offsets[S]) {
            int lo = 0, hi = S;             // offsets[lo] <= row < offsets[hi]
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
                if (E4M3) {
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
    const int64_t blocks = (total + kReadRows - 1) / kReadRows;
    if (blocks > 0x7fffffffLL) {
        set_error("qarl_kv_cache_read: %lld rows exceed the grid limit", (long long)total);
        return QARL_ERR_UNSUPPORTED;
    }
    const dim3 grid((unsigned)blocks), block(kKvThreads);
    uint16_t *ko = (uint16_t *)k_out, *vo = (uint16_t *)v_out;
    const bool e4m3 = c.fmt == QARL_KV_E4M3, nt = total * c.kv_heads * c.head_dim * (e4m3 ? 6 : 8) > kReadCached;
#define QARL_KV_READ(D, E4M3, NT) kv_read_kernel<D, E4M3, NT><<<grid, block, 0, s>>>(c, table, table_stride, table_width, offsets, S, total, ko, vo)
#define QARL_KV_READ_AS(D, E4M3) \
    if (nt) QARL_KV_READ(D, E4M3, true); \
    else QARL_KV_READ(D, E4M3, false)
    if (c.head_dim == 128) {
        if (e4m3) {
            QARL_KV_READ_AS(128, true);
        } else {
            QARL_KV_READ_AS(128, false);
        }
    } else {
        if (e4m3) {
            QARL_KV_READ_AS(64, true);
        } else {
            QARL_KV_READ_AS(64, false);
        }
    }
#undef QARL_KV_READ_AS
#undef QARL_KV_READ
    return check_hip(hipGetLastError(), "kv_read_kernel");
}

}  // namespace qarl
