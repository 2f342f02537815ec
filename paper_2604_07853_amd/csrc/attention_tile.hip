// Attention of many query rows per sequence (prompts, chunks of prompts) over the paged cache.
// Bound by the matrix cores and by exp2.  A workgroup takes a block of 256 rows of one cached head (rows are (query, head of the group)) and runs
// over the cache in tiles of 64 positions, which its eight wavefronts share through two buffers in LDS: while they work on one tile the next one
// arrives (bf16: asynchronous copies; e4m3: through registers, widened to bf16 on the way, once per workgroup).
//
// S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 matrix instructions: a wavefront owns 32 rows, lane (n = lane & 31, half = lane >> 5) holds row n's
// scores at positions 8 (i / 4) + 4 half + i % 4, i = 0 .. 15, of each 32-position tile, so that the maximum and the sum of a row are in-lane
// but for one exchange between the halves, and registers 8 t .. 8 t + 7, packed to bf16, are the B operand of step t of the second product as they
// are (contraction order {4 half + 0..3, 8 + 4 half + 0..3} of 16 positions).  V^T in that order comes out of LDS by transposing reads.
#include "attention.hpp"

namespace qarl {

constexpr int kManyThreads = 64 * kManyWaves;

template <int D>
struct ManyLayout {
    static constexpr int kRowBytes = D * 2, kChunks = kRowBytes / 16;
    static constexpr int kHalf = kManyTile * kRowBytes;              // a tile of keys, or of values
    static constexpr int kScales = 2 * kManyTile * 4;                // e4m3: the tile's key and value scales
    static constexpr int kBuffer = 2 * kHalf + kScales;
    // Chunk c of row r lies at c ^ swz(r).  Keys: 16 rows read at one chunk spread over the banks; values: four rows read at four neighbouring
    // chunks do.
    __device__ static constexpr int swz_k(int r) { return (r / (256 / kRowBytes)) & (kChunks - 1); }
    __device__ static constexpr int swz_v(int r) { return D == 128 ? ((r & 3) << 2 | ((r >> 2) & 3)) : ((r >> 1) & 1) << 2; }
};

template <int D, bool E4M3>
__global__ __launch_bounds__(kManyThreads, 2) void attention_tile_kernel(AttnArgs a, int few_rows, int chunk, int blocks, AttnParts parts)
{
    using L = ManyLayout<D>;
    constexpr int KS = D / 16, DT = D / 32;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m32 = lane & 31, half = lane >> 5;
    const int Hkv = a.kv.kv_heads, G = a.q_heads / Hkv;
    // workgroup -> (piece, row block, cached head), heads fastest: workgroup ids go round the 8 XCDs, so an XCD meets few heads and its L2 keeps them;
    // later row blocks, which see more of the cache, first
    const unsigned per_split = (unsigned)blocks * (unsigned)Hkv;
    const int split = (int)(blockIdx.x / per_split);
    const unsigned bh = blockIdx.x - (unsigned)split * per_split;
    const int h = (int)(bh % (unsigned)Hkv);
    int block = blocks - 1 - (int)(bh / (unsigned)Hkv);
    // the sequence of the row block: 64 sequences at a time, one per lane
    int s = -1;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        int nb = 0;
        if (s0 + lane < a.S) {
            const int lo = max(0, min(a.T, a.q_offsets[s0 + lane])), hi = max(0, min(a.T, a.q_offsets[s0 + lane + 1]));
            const int64_t rows = (int64_t)max(0, hi - lo) * G;
            nb = rows > few_rows ? (int)((rows + kManyRows - 1) / kManyRows) : 0;
        }
        int incl = nb;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int up = __shfl_up(incl, o, 64);
            if (lane >= o) incl += up;
        }
        const unsigned long long hit = __ballot(block < incl);
        if (hit) {
            const int src = __ffsll((long long)hit) - 1;
            s = s0 + src;
            block -= __builtin_amdgcn_readlane(incl, src) - __builtin_amdgcn_readlane(nb, src);
            break;
        }
        block -= __builtin_amdgcn_readlane(incl, 63);
    }
    if (s < 0) return;                                  // the grid is a bound
    const SeqRange sr = seq_range(a, s);
    const int64_t rows = (int64_t)sr.n * G, row0 = (int64_t)block * kManyRows;
    const int in_block = (int)min((int64_t)kManyRows, rows - row0);
    const int i_first = (int)(row0 / G), i_last = (int)((row0 + in_block - 1) / G);
    int begin, end;
    visible_range(a, sr, i_first, i_last, begin, end);
    const int base = begin & ~(kManyTile - 1);
    const int pieces = max(1, (end - base + chunk - 1) / chunk);
    if (split >= pieces) return;
    const int lo = base + split * chunk, hi = min(end, lo + chunk);
    const int tiles = (hi - lo + kManyTile - 1) / kManyTile;
    const int shift = a.kv.page_shift;
    const int32_t *table = a.table + (int64_t)s * a.table_stride;

    // this lane's row: queries as B operand, bounds of what it sees
    const int wrow = wave * 32 + m32;                   // row of the block
    const bool live = wrow < in_block;
    const int64_t row = row0 + (live ? wrow : 0);
    const int qi = (int)(row / G), g = (int)(row - (int64_t)qi * G);
    int see_lo, see_hi;
    row_bounds(a, sr, qi, see_lo, see_hi);
    if (!live) see_hi = -1;
    const int64_t out_row = (int64_t)(sr.row_lo + qi) * a.q_heads + h * G + g;
    bf16x8 qf[KS];
    {
        const uint16_t *qp = (const uint16_t *)a.q + (int64_t)(sr.row_lo + qi) * a.q_token_stride + (int64_t)(h * G + g) * a.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) qf[ks] = __builtin_bit_cast(bf16x8, *(const u32x4 *)(qp + 16 * ks + 8 * half));
    }
    // positions [all_lo, all_hi] are seen by all rows of the wavefront, [any_lo, any_hi] by one at least (a wavefront without rows: none)
    int all_lo, all_hi, any_lo, any_hi;
    {
        const int w_first = (int)((row0 + wave * 32) / G), w_last = (int)((row0 + min(in_block - 1, wave * 32 + 31)) / G);
        row_bounds(a, sr, w_first, any_lo, all_hi);
        row_bounds(a, sr, w_last, all_lo, any_hi);
        if (wave * 32 >= in_block) any_hi = -1;
        any_lo = __builtin_amdgcn_readfirstlane(any_lo);
        any_hi = __builtin_amdgcn_readfirstlane(any_hi);
        all_lo = __builtin_amdgcn_readfirstlane(all_lo);
        all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    }

    // ---- a tile's way into LDS.  A thread moves the same 16-byte chunks (bf16) of every tile: rows kRowsAtOnce apart.
    constexpr int kParts = kManyTile * L::kChunks / kManyThreads;      // 16-byte chunks of keys (and of values) per thread: 2 or 1
    constexpr int kRowsAtOnce = kManyThreads / L::kChunks;
    // e4m3: 16 codes (32 bytes of bf16) of keys and of values per thread; D = 64 keeps half of the threads busy
    constexpr int kCodeChunks = D / 16;
    u32x4 codes[2];
    float scale = 0.f;
    // The page of each of a tile's 64 positions (one per lane), -1 where there is none.  It is requested two tiles ahead: a load behind a tile's
    // copies would wait for them.
    auto find_pages = [&](int t) -> int {
        const int page = table[min(max(lo + t * kManyTile + lane, begin), end - 1) >> shift];
        return page >= 0 && page < a.kv.num_pages ? page : -1;
    };
    // positions outside [begin, end), which may hold anything, are not read: the nearest one inside is, again
    auto in_page = [&](int pos) -> int { return min(max(pos, begin), end - 1) & ((1 << shift) - 1); };
    auto head_page = [&](int page) -> int64_t { return ((int64_t)max(page, 0) * Hkv + h) << shift; };
    auto fetch = [&](int t, int page, char *buf) {
        const int pos0 = lo + t * kManyTile;
        if (!E4M3) {
#pragma unroll
            for (int i = 0; i < kParts; ++i) {      // the rows of a wavefront's copy are 4 or 8 neighbouring positions: one page
                const int r = i * kRowsAtOnce + tid / L::kChunks, pc = tid % L::kChunks;
                const int64_t first = head_page(__builtin_amdgcn_readlane(page, i * kRowsAtOnce + wave * (64 / L::kChunks))) * L::kRowBytes;
                const uint32_t in = (uint32_t)in_page(pos0 + r) * (uint32_t)L::kRowBytes;
                char *to = buf + (i * kManyThreads + wave * 64) * 16;
                copy16_to_lds((const char *)a.kv.k + first + (in + (uint32_t)((pc ^ L::swz_k(r)) * 16)), to);
                copy16_to_lds((const char *)a.kv.v + first + (in + (uint32_t)((pc ^ L::swz_v(r)) * 16)), to + L::kHalf);
            }
        } else {
            const int r = tid / kCodeChunks, c = tid % kCodeChunks;
            if (r < kManyTile) {                    // 8 rows per wavefront (D = 64: 16, two runs of 8)
                constexpr int kPer = 64 / kCodeChunks;
                int pg = __builtin_amdgcn_readlane(page, (wave * kPer) & 63);
                if (kPer > 8 && lane >= 32) pg = __builtin_amdgcn_readlane(page, (wave * kPer + 8) & 63);
                const int64_t at = head_page(pg) * D + (in_page(pos0 + r) * D + c * 16);
                codes[0] = *(const u32x4 *)((const char *)a.kv.k + at);
                codes[1] = *(const u32x4 *)((const char *)a.kv.v + at);
            }
            if (tid < 2 * kManyTile) scale = (tid < kManyTile ? a.kv.k_scales : a.kv.v_scales)[head_page(page) + in_page(pos0 + lane)];
        }
    };
    auto settle = [&](char *buf) {                      // e4m3: the fetched codes as bf16; a value scale that is not finite makes NaN of its row
        if (!E4M3) return;
        const int r = tid / kCodeChunks, c = tid % kCodeChunks;
        if (r < kManyTile) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const bf16x8 x0 = widen_e4m3x8(codes[w][0], codes[w][1]), x1 = widen_e4m3x8(codes[w][2], codes[w][3]);
                char *to = buf + w * L::kHalf + r * L::kRowBytes;
                const int sw = w ? L::swz_v(r) : L::swz_k(r);
                *(bf16x8 *)(to + ((2 * c) ^ sw) * 16) = x0;
                *(bf16x8 *)(to + ((2 * c + 1) ^ sw) * 16) = x1;
            }
        }
        if (tid < 2 * kManyTile) ((float *)(buf + 2 * L::kHalf))[tid] = scale;
    };

    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[dt][e] = 0.f;
    float m = kNegInf, l = 0.f;
    const float c2 = a.scale * kLog2e;

    int pages = -1, pages_next = -1;
    if (tiles > 0) {
        pages = find_pages(0);
        pages_next = find_pages(min(1, tiles - 1));
        asm volatile("" : "+v"(pages), "+v"(pages_next));
        fetch(0, pages, lds);
        settle(lds);
    }
    copy_barrier();
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
        char *buf = lds + (t & 1) * L::kBuffer, *other = lds + (~t & 1) * L::kBuffer;
        int pages_after = find_pages(min(t + 2, tiles - 1));
        if (t + 1 < tiles) fetch(t + 1, pages_next, other);
        const int pos0 = lo + t * kManyTile;
        const unsigned long long holes = __ballot(pages < 0);       // positions without a page are not seen
        if (pos0 <= any_hi && pos0 + kManyTile - 1 >= any_lo) {
            f32x16 z[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
#pragma unroll
                for (int e = 0; e < 16; ++e) z[u][e] = 0.f;
                const int r = u * 32 + m32;
                const char *kr = buf + r * L::kRowBytes;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    z[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const bf16x8 *)(kr + (((2 * ks + half) ^ L::swz_k(r)) * 16)), qf[ks], z[u], 0, 0, 0);
            }
            const float *ks = (const float *)(buf + 2 * L::kHalf), *vs = ks + kManyTile;
            // scores in powers of two
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    f32x4 f = {c2, c2, c2, c2};
                    if (E4M3) f = *(const f32x4 *)(ks + u * 32 + 8 * b + 4 * half) * c2;
#pragma unroll
                    for (int e = 0; e < 4; ++e) z[u][4 * b + e] *= f[e];
                }
            const bool masked = holes != 0 || pos0 < all_lo || pos0 + kManyTile - 1 > all_hi;
            if (masked) {
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int k = u * 32 + 8 * (e >> 2) + 4 * half + (e & 3), j = pos0 + k;
                        if (!(j >= see_lo && j <= see_hi) || (holes >> k & 1ull)) z[u][e] = kNegInf;
                    }
            }
            float mx = z[0][0];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = fmaxf(mx, z[u][e]);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            if (__ballot(mx > m + kStale) != 0) {
                const float to = mx > m + kStale ? mx : m;       // a row goes by its own scores alone
                const float keep = to == kNegInf ? 1.f : __builtin_amdgcn_exp2f(m - to);
                m = to;
                l *= keep;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) acc[dt] *= keep;
            }
            const float mb = m == kNegInf ? 0.f : m;
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    z[u][e] = __builtin_amdgcn_exp2f(z[u][e] - mb);
                    sum += z[u][e];
                }
            l += sum;
            // V^T of step t16 (16 positions), 32 of D: lanes of a block of 16 name the rows and columns that the block transposes
            auto frag = [&](int t16, int dt) -> bf16x8 {
                union {
                    s16x4 part[2];
                    bf16x8 v;
                } f;
                const int i16 = lane & 15, dh = (lane >> 4) & 1;
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int r = 16 * t16 + 8 * p + 4 * half + (i16 >> 2);
                    const int c = 4 * dt + 2 * dh + ((i16 & 3) >> 1);
                    f.part[p] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4 *)(buf + L::kHalf + r * L::kRowBytes + ((c ^ L::swz_v(r)) * 16) + (i16 & 1) * 8));
                }
                return f.v;
            };
            bool rare = false;
            if (masked) {       // a value that a row does not see may be an infinity or a NaN
                uint32_t seen = 0;
#pragma unroll
                for (int t16 = 0; t16 < 4; ++t16)
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        const u32x4 w = __builtin_bit_cast(u32x4, frag(t16, dt));
#pragma unroll
                        for (int e = 0; e < 4; ++e) seen = gather_nonfinite(seen, w[e]);
                    }
                bool bad = any_nonfinite(seen);
                if (E4M3) bad |= !(fabsf(vs[lane]) < __builtin_inff());
                rare = __ballot(bad) != 0;
            }
            if (!rare) {
#pragma unroll
                for (int t16 = 0; t16 < 4; ++t16) {
                    float p[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) p[e] = z[t16 >> 1][8 * (t16 & 1) + e];
                    if (E4M3) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            const f32x4 f = *(const f32x4 *)(vs + 16 * t16 + 8 * b + 4 * half);
#pragma unroll
                            for (int e = 0; e < 4; ++e) p[4 * b + e] *= f[e];
                        }
                    }
                    const bf16x8 pf = pack_bf16x8(p);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag(t16, dt), pf, acc[dt], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int t16 = 0; t16 < 4; ++t16) {
                    float p[8], one[8], sc[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        p[e] = z[t16 >> 1][8 * (t16 & 1) + e];
                        one[e] = p[e] == 0.f ? 0.f : 1.f;           // (a NaN counts as seen)
                        sc[e] = 1.f;
                        if (E4M3) {
                            sc[e] = vs[16 * t16 + 8 * (e >> 2) + 4 * half + (e & 3)];
                            p[e] = fabsf(sc[e]) < __builtin_inff() ? p[e] * sc[e] : 0.f;
                        }
                    }
                    const bf16x8 pf = pack_bf16x8(p), see = pack_bf16x8(one);
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        u32x4 w = __builtin_bit_cast(u32x4, frag(t16, dt));
                        if (E4M3) {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (!(fabsf(sc[e]) < __builtin_inff())) w[e >> 1] |= 0x7fc0u << (16 * (e & 1));
                        }
                        bf16x8 fine, up, down;
                        split_nonfinite(__builtin_bit_cast(bf16x8, w), fine, up, down);
                        f32x16 none;
#pragma unroll
                        for (int e = 0; e < 16; ++e) none[e] = 0.f;
                        const f32x16 ups = __builtin_amdgcn_mfma_f32_32x32x16_bf16(up, see, none, 0, 0, 0);
                        const f32x16 downs = __builtin_amdgcn_mfma_f32_32x32x16_bf16(down, see, none, 0, 0, 0);
                        acc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fine, pf, acc[dt], 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[dt][e] += (ups[e] > 0.f ? __builtin_inff() : 0.f) + (downs[e] > 0.f ? kNegInf : 0.f);
                    }
                }
            }
        }
        if (t + 1 < tiles) settle(other);
        copy_barrier();
        asm volatile("" : "+v"(pages_after));
        pages = pages_next;
        pages_next = pages_after;
    }
    l += __shfl_xor(l, 32, 64);
    if (!live) return;
    // lane (row n, half) holds D index 32 dt + 8 (e / 4) + 4 half + e % 4
    const float inv = inverse_sum(l);
    float *po = parts.o + ((int64_t)split * parts.rows + out_row) * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            f32x4 o = {acc[dt][4 * b], acc[dt][4 * b + 1], acc[dt][4 * b + 2], acc[dt][4 * b + 3]};
            const int d = 32 * dt + 8 * b + 4 * half;
            if (pieces == 1) store_out4(a, out_row, D, d, o * inv);
            else *(f32x4 *)(po + d) = o;
        }
    if (half == 0) {
        if (pieces == 1) {
            if (a.lse) a.lse[out_row] = (m + __builtin_amdgcn_logf(l)) * kLn2;
        } else {
            parts.ml[((int64_t)split * parts.rows + out_row) * 2] = m;
            parts.ml[((int64_t)split * parts.rows + out_row) * 2 + 1] = l;
        }
        if (split == 0 && parts.splits > 0) parts.count[out_row] = pieces;
    }
}

template <int D, bool E4M3>
static int launch_tile_as(const AttnArgs &a, const AttnPlan &p, const AttnParts &parts, hipStream_t s)
{
    static LdsLimitOnce once;
    const int64_t grid = (int64_t)p.tile_blocks * a.kv.kv_heads * p.tile_splits;
    if (grid > 0x7fffffffLL) {
        set_error("qarl_paged_attention: %lld row blocks exceed the grid limit", (long long)grid);
        return QARL_ERR_UNSUPPORTED;
    }
    int rc = raise_lds_limit((const void *)attention_tile_kernel<D, E4M3>, once, "attention_tile_kernel");
    if (rc) return rc;
    attention_tile_kernel<D, E4M3><<<dim3((unsigned)grid), dim3(kManyThreads), 2 * ManyLayout<D>::kBuffer, s>>>(a, 16 * p.few_nr, p.tile_chunk, p.tile_blocks, parts);
    return check_hip(hipGetLastError(), "attention_tile_kernel");
}

int launch_attention_tile(const AttnArgs &a, const AttnPlan &p, const AttnParts &parts, hipStream_t s)
{
    const bool e4m3 = a.kv.fmt == QARL_KV_E4M3;
    if (a.kv.head_dim == 128) return e4m3 ? launch_tile_as<128, true>(a, p, parts, s) : launch_tile_as<128, false>(a, p, parts, s);
    return e4m3 ? launch_tile_as<64, true>(a, p, parts, s) : launch_tile_as<64, false>(a, p, parts, s);
}

}  // namespace qarl
