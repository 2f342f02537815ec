// Attention of few query rows per sequence (single tokens, a few speculated ones) over the paged cache.
// Bound by memory: G query heads share a cached one, 4 G D operations per 4 D bytes.  A workgroup takes one (sequence, cached head, piece
// of the cache); its four wavefronts take every fourth tile of 32 positions each, with running maxima and sums of their own, which they
// join at the end.  (32 query heads on 4 of 128, 256 sequences of 4096 positions: bf16 361 us, 6.0 TB/s, e4m3 196 us, 5.7; 256 of up to 18432 e4m3 453 us, 5.3; one of 18432, where
// lengths, pages and keys wait for one another, 10.6 us.)  Keys and values flow through rings in LDS, private to a wavefront and filled by asynchronous copies, so that a wavefront waits
// for its own copies only and no barrier stands in the loop.
//
// S^T = K Q^T and O^T = V^T P^T on 16 x 16 x 32 matrix instructions: lane (n = lane & 15, q = lane >> 4) then holds the scores of row n at
// positions 4 q + i of a 16-position tile, which are, packed to bf16, the B operand of the second product as they are, if its contraction
// runs over positions in the order {4 q + 0..3, 16 + 4 q + 0..3}.  V^T in that order comes out of LDS by transposing reads.
#include "attention.hpp"

namespace qarl {

constexpr int kFewWaves = 4, kFewThreads = 64 * kFewWaves;

template <int D, bool E4M3>
struct FewLayout {
    static constexpr int kRowBytes = D * (E4M3 ? 1 : 2);
    static constexpr int kChunks = kRowBytes / 16;                       // 16-byte chunks of a row
    static constexpr int kRowsPerCopy = 1024 / kRowBytes;                // an asynchronous copy moves 64 x 16 bytes
    static constexpr int kCopies = kFewTile / kRowsPerCopy;              // per tile of keys, and of values
    static constexpr int kHalf = kFewTile * kRowBytes;                   // bytes of a tile of keys
    static constexpr int kStage = 2 * kHalf + (E4M3 ? 256 : 0);          // keys, values, 32 + 32 scales
    static constexpr int kStageCopies = 2 * kCopies + (E4M3 ? 1 : 0);
    static constexpr int kRing = kStage <= 5000 ? 4 : 2;                 // stages; about 64 KiB per workgroup, D = 128 in bf16 128
    // Chunk c of row r lies at chunk c ^ swz(r): 16 rows that are read at the same chunk spread over all banks
    __device__ static constexpr int swz(int r) { return (r / (256 / kRowBytes)) & (kChunks - 1); }
};

template <int D, bool E4M3, int NR>
__global__ __launch_bounds__(kFewThreads, NR == 4 ? 1 : 2) void attention_few_kernel(AttnArgs a, int chunk, AttnParts parts)
{
    using L = FewLayout<D, E4M3>;
    constexpr int KS = D / 32, DT = D / 16;
    extern __shared__ __align__(16) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m16 = lane & 15, q = lane >> 4;
    const int Hkv = a.kv.kv_heads, G = a.q_heads / Hkv;
    const unsigned per_split = (unsigned)a.S * (unsigned)Hkv;
    const int split = (int)(blockIdx.x / per_split);
    const unsigned sh = blockIdx.x - (unsigned)split * per_split;
    const int s = (int)(sh / (unsigned)Hkv), h = (int)(sh - (unsigned)s * (unsigned)Hkv);
    const SeqRange sr = seq_range(a, s);
    if (over_long(a, sr)) {
        if (split == 0 && parts.splits > 0) {
            for (int64_t i = tid; i < (int64_t)sr.n * G; i += kFewThreads) parts.count[(sr.row_lo + i / G) * a.q_heads + h * G + i % G] = 0;
        }
        return;
    }
    if (sr.n == 0 || (int64_t)sr.n * G > 16 * NR) return;
    const int R = sr.n * G;
    int begin, end;
    visible_range(a, sr, 0, sr.n - 1, begin, end);
    const auto [base, pieces] = cut_range(begin, end, kFewTile, chunk);
    if (split >= pieces) return;
    const int lo = base + split * chunk, hi = min(end, lo + chunk);      // this piece; lo is a multiple of 32
    const int tiles = (hi - lo + kFewTile - 1) / kFewTile;               // (0 where nothing is visible)
    const int shift = a.kv.page_shift;

    char *ring = lds + wave * (L::kRing * L::kStage);
    int *pages = (int *)(lds + kFewWaves * L::kRing * L::kStage);        // page of every eight positions of the piece, -1: none
    const int32_t *table = a.table + (int64_t)s * a.table_stride;
    for (int i = tid; i < tiles * (kFewTile / 8); i += kFewThreads) {
        const int pos = min(max(lo + 8 * i, begin), end - 1);            // positions outside are the nearest one's again
        const int page = table[pos >> shift];
        pages[i] = page >= 0 && page < a.kv.num_pages ? page : -1;
    }
    // the queries: B operand, lane holds row n = lane & 15, eight of D at 8 q (bf16 cache) or as the keys' 16-byte reads order them (e4m3)
    bf16x8 qf[NR][KS];
    int see_lo[NR], see_hi[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        const int row = r * 16 + m16, i = row < R ? row / G : 0, g = row - i * G;
        row_bounds(a, sr, i, see_lo[r], see_hi[r]);
        const uint16_t *qp = (const uint16_t *)a.q + (int64_t)(sr.row_lo + i) * a.q_token_stride + (int64_t)(h * G + (row < R ? g : 0)) * a.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int d = E4M3 ? 64 * (ks >> 1) + 16 * q + 8 * (ks & 1) : 32 * ks + 8 * q;
            qf[r][ks] = __builtin_bit_cast(bf16x8, *(const u32x4 *)(qp + d));
        }
        if (row >= R) see_hi[r] = -1;
    }
#pragma unroll
    for (int r = 0; r < NR; ++r)
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[r][ks]));   // here before copies are in flight (a later wait would include them)
    lds_barrier();

    // Copies of tile t into a stage.  Eight neighbouring positions lie in one page; positions outside [begin, end), which may hold
    // anything, are not read: the nearest position inside is, again.
    auto fill = [&](int t, int slot) {
        char *to = ring + slot * L::kStage;
        const int pos0 = lo + t * kFewTile;
        const int pl = pages[t * 4 + ((lane & 31) >> 3)];
        // rows of a copy: lane / kChunks-th position, 16 bytes each
#pragma unroll
        for (int c = 0; c < L::kCopies; ++c) {
            const int r = c * L::kRowsPerCopy + lane / L::kChunks;
            const int logical = (lane % L::kChunks) ^ L::swz(r);
            int page;
            if (L::kRowsPerCopy <= 8) page = __builtin_amdgcn_readlane(pl, c * L::kRowsPerCopy);
            else page = lane < 32 ? __builtin_amdgcn_readlane(pl, c * 16) : __builtin_amdgcn_readlane(pl, c * 16 + 8);
            const int64_t first = ((int64_t)max(page, 0) * Hkv + h) << shift;
            const uint32_t in = (uint32_t)(min(max(pos0 + r, begin), end - 1) & ((1 << shift) - 1)) * (uint32_t)L::kRowBytes + (uint32_t)(logical * 16);
            copy16_to_lds((const char *)a.kv.k + first * L::kRowBytes + in, to + c * 1024);
            copy16_to_lds((const char *)a.kv.v + first * L::kRowBytes + in, to + L::kHalf + c * 1024);
        }
        if (E4M3) {
            const int64_t at = (((int64_t)max(pl, 0) * Hkv + h) << shift) + (min(max(pos0 + (lane & 31), begin), end - 1) & ((1 << shift) - 1));
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)((lane < 32 ? a.kv.k_scales : a.kv.v_scales) + at),
                                             (__attribute__((address_space(3))) void *)(to + 2 * L::kHalf), 4, 0, 0);
        }
    };

    f32x4 acc[NR][DT];
    float m[NR], l[NR];
#pragma unroll
    for (int r = 0; r < NR; ++r) {
        m[r] = kNegInf;
        l[r] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) acc[r][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float c2 = a.scale * kLog2e;
    // positions [all_lo, all_hi] are seen by every row
    int all_lo, all_hi, unused;
    row_bounds(a, sr, 0, unused, all_hi);
    row_bounds(a, sr, sr.n - 1, all_lo, unused);

    bool rare = false;      // values that are not finite were found in a tile that some row does not see whole
    const int mine = tiles > wave ? (tiles - wave + kFewWaves - 1) / kFewWaves : 0;
#pragma unroll
    for (int i = 0; i < L::kRing - 1; ++i)
        if (i < mine) fill(wave + i * kFewWaves, i);
    int slot = 0;
#pragma unroll 1
    for (int i = 0; i < mine; ++i) {
        const int t = wave + i * kFewWaves;
        if (i + L::kRing - 1 < mine) {
            int ahead = slot + L::kRing - 1;
            ahead = ahead >= L::kRing ? ahead - L::kRing : ahead;
            fill(t + (L::kRing - 1) * kFewWaves, ahead);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(L::kStageCopies * (L::kRing - 1)) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        const char *st = ring + slot * L::kStage;
        const int pos0 = lo + t * kFewTile;
        // ---- scores
        f32x4 z[2][NR];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int r = u * 16 + m16;
#pragma unroll
            for (int n = 0; n < NR; ++n) z[u][n] = f32x4{0.f, 0.f, 0.f, 0.f};
            const char *kr = st + r * L::kRowBytes;
            if (E4M3) {
#pragma unroll
                for (int kp = 0; kp < KS / 2; ++kp) {
                    const u32x4 w = *(const u32x4 *)(kr + (((4 * kp + q) ^ L::swz(r)) * 16));
                    const bf16x8 k0 = widen_e4m3x8(w[0], w[1]), k1 = widen_e4m3x8(w[2], w[3]);
#pragma unroll
                    for (int n = 0; n < NR; ++n) {
                        z[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k0, qf[n][2 * kp], z[u][n], 0, 0, 0);
                        z[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k1, qf[n][2 * kp + 1], z[u][n], 0, 0, 0);
                    }
                }
            } else {
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const bf16x8 k = *(const bf16x8 *)(kr + (((4 * ks + q) ^ L::swz(r)) * 16));
#pragma unroll
                    for (int n = 0; n < NR; ++n) z[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, qf[n][ks], z[u][n], 0, 0, 0);
                }
            }
        }
        f32x4 vs[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            f32x4 kscale = f32x4{c2, c2, c2, c2};
            if (E4M3) {
                kscale = *(const f32x4 *)(st + 2 * L::kHalf + (u * 16 + 4 * q) * 4) * c2;
                vs[u] = *(const f32x4 *)(st + 2 * L::kHalf + 128 + (u * 16 + 4 * q) * 4);
            }
#pragma unroll
            for (int n = 0; n < NR; ++n) z[u][n] *= kscale;
        }
        // ---- masks: tiles that not every row sees whole
        const int pl = pages[t * 4 + ((lane & 31) >> 3)];
        const bool holes = __ballot(pl < 0) != 0;
        const bool masked = holes || pos0 < all_lo || pos0 + kFewTile - 1 > all_hi;
        if (masked) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool page_ok = pages[t * 4 + u * 2 + (q >> 1)] >= 0;
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int j = pos0 + u * 16 + 4 * q + e;
                        if (!(page_ok && j >= see_lo[n] && j <= see_hi[n])) z[u][n][e] = kNegInf;
                    }
            }
        }
        // ---- running maximum and sum
        bf16x8 pf[NR];
        float pv[NR][8];
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            float mx = fmaxf(fmaxf(fmaxf(z[0][n][0], z[0][n][1]), fmaxf(z[0][n][2], z[0][n][3])),
                             fmaxf(fmaxf(z[1][n][0], z[1][n][1]), fmaxf(z[1][n][2], z[1][n][3])));
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            if (__ballot(mx > m[n] + kStale) != 0) {
                const float to = mx > m[n] + kStale ? mx : m[n];       // a row goes by its own scores alone
                const float keep = to == kNegInf ? 1.f : __builtin_amdgcn_exp2f(m[n] - to);
                m[n] = to;
                l[n] *= keep;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) acc[n][dt] *= keep;
            }
            const float mb = m[n] == kNegInf ? 0.f : m[n];
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                pv[n][e] = __builtin_amdgcn_exp2f(z[e >> 2][n][e & 3] - mb);
                sum += pv[n][e];
            }
            l[n] += sum;
        }
        // ---- values.  Where rows see different positions (or a page is missing), a value that one of them does not see may be an infinity or a NaN,
        // and its product with the probability 0 a NaN: such values become zeros in LDS, and the rows that see them get them in the end.  (For single
        // tokens too: what lies outside the positions that they see was read from the nearest of those.)
        if (masked) {
            bool bad = false;
#pragma unroll
            for (int i = 0; i < L::kHalf / 1024; ++i) {
                u32x4 *w = (u32x4 *)(ring + slot * L::kStage + L::kHalf) + i * 64 + lane;
                u32x4 v = *w;
                const u32x4 was = v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = E4M3 ? only_finite_e4m3(v[e]) : only_finite_bf16(v[e]);
                if (v[0] != was[0] || v[1] != was[1] || v[2] != was[2] || v[3] != was[3]) {
                    *w = v;
                    bad = true;
                }
            }
            if (E4M3) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(fabsf(vs[e >> 2][e & 3]) < __builtin_inff())) {
                        vs[e >> 2][e & 3] = 0.f;
                        bad = true;
                    }
            }
            rare |= __ballot(bad) != 0;
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            if (E4M3) {
#pragma unroll
                for (int e = 0; e < 8; ++e) pv[n][e] *= vs[e >> 2][e & 3];
            }
            pf[n] = pack_bf16x8(pv[n]);
        }
        // (the reads and their wait in one block: the compiler would let a transposing read that it can see wait for the copies in flight)
#pragma unroll
        for (int d4 = 0; d4 < DT; d4 += 4) {
            bf16x8 v[4];
            if (E4M3) {
                const int r = ((m16 >> 1) & 3) + 4 * q + 16 * (m16 >> 3);
                const uint32_t at = (uint32_t)(uintptr_t)(LdsPtr)st + L::kHalf + r * L::kRowBytes + (L::swz(r) * 16) + (m16 & 1) * 8;
                u32x2 w[4];
                asm volatile("ds_read_b64_tr_b8 %0, %4\n\tds_read_b64_tr_b8 %1, %5\n\tds_read_b64_tr_b8 %2, %6\n\tds_read_b64_tr_b8 %3, %7\n\t"
                             "s_waitcnt lgkmcnt(0)"
                             : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3])
                             : "v"(at ^ (d4 * 16)), "v"(at ^ (d4 * 16 + 16)), "v"(at ^ (d4 * 16 + 32)), "v"(at ^ (d4 * 16 + 48))
                             : "memory");
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = widen_e4m3x8(w[x][0], w[x][1]);
            } else {
                const int r = 4 * q + (m16 >> 2);
                const uint32_t at = (uint32_t)(uintptr_t)(LdsPtr)st + L::kHalf + r * L::kRowBytes + ((((m16 & 3) >> 1) ^ L::swz(r)) * 16) + (m16 & 1) * 8;
                static_assert(E4M3 || L::swz(16) == 0, "positions 16 apart lie at the same chunk");
                u32x2 w[8];
                asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\tds_read_b64_tr_b16 %2, %9\n\t"
                             "ds_read_b64_tr_b16 %3, %9 offset:%12\n\tds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
                             "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\ts_waitcnt lgkmcnt(0)"
                             : "=&v"(w[0]), "=&v"(w[1]), "=&v"(w[2]), "=&v"(w[3]), "=&v"(w[4]), "=&v"(w[5]), "=&v"(w[6]), "=&v"(w[7])
                             : "v"(at ^ (d4 * 32)), "v"(at ^ (d4 * 32 + 32)), "v"(at ^ (d4 * 32 + 64)), "v"(at ^ (d4 * 32 + 96)), "n"(16 * L::kRowBytes)
                             : "memory");
#pragma unroll
                for (int x = 0; x < 4; ++x) v[x] = __builtin_bit_cast(bf16x8, u32x4{w[2 * x][0], w[2 * x][1], w[2 * x + 1][0], w[2 * x + 1][1]});
            }
#pragma unroll
            for (int x = 0; x < 4; ++x)
#pragma unroll
                for (int n = 0; n < NR; ++n) acc[n][d4 + x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[x], pf[n], acc[n][d4 + x], 0, 0, 0);
        }
        slot = slot == L::kRing - 1 ? 0 : slot + 1;
    }

    if (rare) {
#pragma unroll 1
        for (int i = 0; i < mine; ++i) {
            const int t = wave + i * kFewWaves, pos0 = lo + t * kFewTile;
            const bool holes = __ballot(pages[t * 4 + ((lane & 31) >> 3)] < 0) != 0;
            if (!holes && pos0 >= all_lo && pos0 + kFewTile - 1 <= all_hi) continue;
            for (int j = max(pos0, begin); j < min(pos0 + kFewTile, end); ++j) {
                const int page = pages[(j - lo) >> 3];
                if (page < 0) continue;
                const int64_t at = (((int64_t)page * Hkv + h) << shift) + (j & ((1 << shift) - 1));
                const float sc = E4M3 ? a.kv.v_scales[at] : 1.f;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int64_t d = at * D + 16 * dt + 4 * q + e;
                        const float v = E4M3 ? sc * __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)a.kv.v)[d], 0) : bf16_bits_to_f32(((const uint16_t *)a.kv.v)[d]);
                        const bool bad = !(fabsf(v) < __builtin_inff());
#pragma unroll
                        for (int n = 0; n < NR; ++n)
                            if (bad && j >= see_lo[n] && j <= see_hi[n]) acc[n][dt][e] += v;
                    }
            }
        }
    }
    // ---- the wavefronts' results meet in LDS (the ring's place; no copy is in flight any more)
    constexpr int kStride = D + 4;
    float *so = (float *)lds;                                             // [wave][16 NR][kStride]
    float *sml = so + kFewWaves * 16 * NR * kStride;                      // [wave][16 NR][2]
    __syncthreads();
#pragma unroll
    for (int n = 0; n < NR; ++n) {
        l[n] += __shfl_xor(l[n], 16, 64);
        l[n] += __shfl_xor(l[n], 32, 64);
        const int row = wave * 16 * NR + n * 16 + m16;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) *(f32x4 *)(so + row * kStride + 16 * dt + 4 * q) = acc[n][dt];
        if (q == 0) {
            sml[row * 2] = m[n];
            sml[row * 2 + 1] = l[n];
        }
    }
    __syncthreads();
    for (int i = tid; i < R * (D / 4); i += kFewThreads) {
        const int row = i / (D / 4), d = (i - row * (D / 4)) * 4;
        float mw[kFewWaves], top = kNegInf;
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            mw[w] = sml[(w * 16 * NR + row) * 2];
            top = fmaxf(top, mw[w]);
        }
        const float tb = top == kNegInf ? 0.f : top;
        float sum = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(mw[w] - tb);
            sum += f * sml[(w * 16 * NR + row) * 2 + 1];
            o += *(const f32x4 *)(so + (w * 16 * NR + row) * kStride + d) * f;
        }
        const int64_t qi = row / G;
        const int64_t out_row = (sr.row_lo + qi) * a.q_heads + h * G + (row - qi * G);
        if (pieces == 1) {
            store_out4(a, out_row, D, d, o * inverse_sum(sum));
            if (d == 0 && a.lse) a.lse[out_row] = (top + __builtin_amdgcn_logf(sum)) * kLn2;
        } else {
            *(f32x4 *)(parts.o + ((int64_t)split * parts.rows + out_row) * D + d) = o;
            if (d == 0) {
                parts.ml[((int64_t)split * parts.rows + out_row) * 2] = top;
                parts.ml[((int64_t)split * parts.rows + out_row) * 2 + 1] = sum;
            }
        }
        if (d == 0 && split == 0 && parts.splits > 0) parts.count[out_row] = pieces;
    }
}

template <int D, bool E4M3, int NR>
static int launch_few_as(const AttnArgs &a, const AttnPlan &p, const AttnParts &parts, hipStream_t s)
{
    using L = FewLayout<D, E4M3>;
    static LdsLimitOnce once;
    const int64_t grid = (int64_t)a.S * a.kv.kv_heads * p.few_splits;
    if (grid > 0x7fffffffLL) {
        set_error("qarl_paged_attention: %lld pieces exceed the grid limit", (long long)grid);
        return QARL_ERR_UNSUPPORTED;
    }
    const int stream = kFewWaves * L::kRing * L::kStage + p.few_chunk / 8 * 4, join = kFewWaves * 16 * NR * (D + 4 + 2) * 4;
    int rc = raise_lds_limit((const void *)attention_few_kernel<D, E4M3, NR>, once, "attention_few_kernel");
    if (rc) return rc;
    attention_few_kernel<D, E4M3, NR><<<dim3((unsigned)grid), dim3(kFewThreads), stream > join ? stream : join, s>>>(a, p.few_chunk, parts);
    return check_hip(hipGetLastError(), "attention_few_kernel");
}

template <int D, bool E4M3>
static int launch_few_rows(const AttnArgs &a, const AttnPlan &p, const AttnParts &parts, hipStream_t s)
{
    if (p.few_nr == 1) return launch_few_as<D, E4M3, 1>(a, p, parts, s);
    if (p.few_nr == 2) return launch_few_as<D, E4M3, 2>(a, p, parts, s);
    return launch_few_as<D, E4M3, 4>(a, p, parts, s);
}

int launch_attention_few(const AttnArgs &a, const AttnPlan &p, const AttnParts &parts, hipStream_t s)
{
    const bool e4m3 = a.kv.fmt == QARL_KV_E4M3;
    if (a.kv.head_dim == 128) return e4m3 ? launch_few_rows<128, true>(a, p, parts, s) : launch_few_rows<128, false>(a, p, parts, s);
    return e4m3 ? launch_few_rows<64, true>(a, p, parts, s) : launch_few_rows<64, false>(a, p, parts, s);
}

}  // namespace qarl
