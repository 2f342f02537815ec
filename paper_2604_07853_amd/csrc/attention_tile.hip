// Attention of many query rows per sequence (prompts, chunks of prompts) over the paged cache.
// Bound by the matrix cores and exp2.  A workgroup takes a block of 256 rows of one cached head (rows are (query, head of the group)) and runs over the
// cache in tiles of 64 positions, which its four wavefronts share through rings of three tiles in LDS.
//
// S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 matrix instructions: a wavefront owns 64 rows, two sets of 32, so that every fragment read from LDS
// feeds two instructions (with 32 rows the LDS reads alone would take as long as the products: 1.1 us per 256 rows and tile).  Lane (n = lane & 31,
// half = lane >> 5) holds row n's scores at positions 8 (i / 4) + 4 half + i % 4, i = 0 .. 15, of 32 positions: the maximum and the sum of a row are
// in-lane but for one exchange between the halves, and registers 8 t .. 8 t + 7, packed to bf16, are the B operand of step t of the second product as
// they are (contraction order {4 half + 0..3, 8 + 4 half + 0..3} of 16 positions).  V^T in that order comes out of LDS by transposing reads.
//
// That takes the registers of a whole SIMD (one wavefront each), so what overlaps is one wavefront's own work: step s (32 positions) computes the scores
// of step s + 1 and adds the values of step s - 1 on the matrix cores while the vector units turn the scores of step s into probabilities; none of the three
// waits for another.
#include "attention.hpp"

namespace qarl {

constexpr int kManyThreads = 64 * kManyWaves;

// Tiles lie in LDS in bf16, whatever the cache holds (e4m3 codes are widened once per workgroup, on their way).
template <int D>
struct ManyLayout {
    static constexpr int kRowBytes = D * 2, kChunks = kRowBytes / 16;
    static constexpr int kHalf = kManyTile * kRowBytes;              // a tile of keys, or of values
    static constexpr int kRing = 3;
    static constexpr int kScale = kManyTile * 4;                     // e4m3: a tile's scales of keys, or of values
    static constexpr int kLds = kRing * 2 * (kHalf + kScale) + 16;   // keys, values, their scales, a flag
    // Chunk c of row r lies at c ^ swz(r), so that the rows that one read touches at the same chunk spread over the banks
    __device__ static constexpr int swz_k(int r) { return (r / (256 / kRowBytes)) & (kChunks - 1); }
    __device__ static constexpr int swz_v(int r) { return D == 128 ? ((r & 3) << 2 | ((r >> 2) & 3)) : ((r >> 1) & 1) << 2; }
};

template <int D, bool E4M3>
__global__ __launch_bounds__(kManyThreads, 2) void attention_tile_kernel(AttnArgs a, int few_rows, int chunk, int blocks, AttnParts parts)
{
    using L = ManyLayout<D>;
    constexpr int KS = D / 16, DT = D / 32, NR = kManyRows / kManyWaves / 32;      // sets of 32 rows per wavefront
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

    // this lane's two rows: queries as B operand, bounds of what they see
    bf16x8 qf[NR][KS];
    int see_lo[NR], see_hi[NR];
#pragma unroll
    for (int rh = 0; rh < NR; ++rh) {
        const int in_rows = (wave * NR + rh) * 32 + m32;
        const int64_t row = row0 + (in_rows < in_block ? in_rows : 0);
        const int qi = (int)(row / G), g = (int)(row - (int64_t)qi * G);
        row_bounds(a, sr, qi, see_lo[rh], see_hi[rh]);
        if (in_rows >= in_block) see_hi[rh] = -1;
        const uint16_t *qp = (const uint16_t *)a.q + (int64_t)(sr.row_lo + qi) * a.q_token_stride + (int64_t)(h * G + g) * a.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            u32x4 w = *(const u32x4 *)(qp + 16 * ks + 8 * half);
            if (a.scale < 0.f) w ^= 0x80008000u;        // scores go by the scale's size: the running maximum wants it positive
            qf[rh][ks] = __builtin_bit_cast(bf16x8, w);
        }
    }
    const float c2 = fmaxf(fabsf(a.scale) * kLog2e, 1e-30f), stale = kStale / c2;
    // positions [all_lo, all_hi] are seen by all rows of the wavefront, [any_lo, any_hi] by one at least (a wavefront without rows: none)
    int all_lo, all_hi, any_lo, any_hi;
    {
        const int w_first = (int)((row0 + wave * 32 * NR) / G), w_last = (int)((row0 + min(in_block - 1, wave * 32 * NR + 32 * NR - 1)) / G);
        row_bounds(a, sr, w_first, any_lo, all_hi);
        row_bounds(a, sr, w_last, all_lo, any_hi);
        if (wave * 32 * NR >= in_block) any_hi = -1;
        any_lo = __builtin_amdgcn_readfirstlane(any_lo);
        any_hi = __builtin_amdgcn_readfirstlane(any_hi);
        all_lo = __builtin_amdgcn_readfirstlane(all_lo);
        all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    }

    // and [blk_lo, blk_hi] by all rows of the block
    int blk_lo, blk_hi, unused;
    row_bounds(a, sr, i_first, unused, blk_hi);
    row_bounds(a, sr, i_last, blk_lo, unused);

    // ---- LDS: three tiles of keys, three of values, their scales, a flag
    char *const lds_k = lds, *const lds_v = lds + L::kRing * L::kHalf, *const lds_s = lds + 2 * L::kRing * L::kHalf;
    int *const lds_flag = (int *)(lds_s + L::kRing * 2 * L::kScale);
    // The page of each of a tile's 64 positions (one per lane), -1 where there is none.  It is requested well ahead: a load behind a tile's
    // copies would wait for them.
    auto find_pages = [&](int t) -> int {
        const int page = table[min(max(lo + min(t, tiles - 1) * kManyTile + lane, begin), end - 1) >> shift];
        return page >= 0 && page < a.kv.num_pages ? page : -1;
    };
    // positions outside [begin, end), which may hold anything, are not read: the nearest one inside is, again
    auto in_page = [&](int pos) -> int { return min(max(pos, begin), end - 1) & ((1 << shift) - 1); };
    auto head_page = [&](int page) -> int64_t { return ((int64_t)max(page, 0) * Hkv + h) << shift; };
    // ---- a tile's way from the cache through registers into LDS.  A thread moves 16-byte pieces, kStep positions apart; the 4, 8 or 16 neighbouring
    // positions of a wavefront's load lie in one page, or each eight of them do.  (Asynchronous copies into LDS would make the compiler wait for all of
    // them in front of every transposing read.)
    constexpr int kPieces = D * (E4M3 ? 1 : 2) / 16;                   // 16-byte pieces of a row of the cache
    constexpr int kPer = 64 / kPieces, kLoads = kManyTile * kPieces > kManyThreads ? kManyTile * kPieces / kManyThreads : 1, kStep = kManyWaves * kPer;
    constexpr bool kHalfBusy = kManyTile * kPieces < kManyThreads;     // (e4m3, D = 64: four of the eight wavefronts)
    const int r_first = wave * kPer + lane / kPieces, piece = lane % kPieces;
    struct Staged {
        u32x4 w[kLoads];
        float scale;
    };
    auto load = [&](const void *from, const float *scales, int t, int page, int scale_wave, Staged &st) {
        const int pos0 = lo + t * kManyTile;
        if (!kHalfBusy || r_first < kManyTile) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int first = (i * kStep + wave * kPer) & (kManyTile - 1);
                int pg = __builtin_amdgcn_readlane(page, first);
                if (kPer > 8) {
                    const int second = __builtin_amdgcn_readlane(page, first + 8);
                    pg = lane < 32 ? pg : second;
                }
                const uint32_t in = (uint32_t)in_page(pos0 + r_first + i * kStep) * (uint32_t)(kPieces * 16) + (uint32_t)(piece * 16);
                st.w[i] = *(const u32x4 *)((const char *)from + head_page(pg) * (kPieces * 16) + in);
            }
        }
        if (E4M3 && wave == scale_wave) st.scale = scales[head_page(page) + in_page(pos0 + lane)];
    };
    auto store = [&](bool is_v, int slot, int scale_wave, const Staged &st) {
        char *to = (is_v ? lds_v : lds_k) + slot * L::kHalf;
        if (!kHalfBusy || r_first < kManyTile) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = r_first + i * kStep, sw = is_v ? L::swz_v(r) : L::swz_k(r);
                if (E4M3) {
                    *(bf16x8 *)(to + r * L::kRowBytes + (((2 * piece) ^ sw) * 16)) = widen_e4m3x8(st.w[i][0], st.w[i][1]);
                    *(bf16x8 *)(to + r * L::kRowBytes + (((2 * piece + 1) ^ sw) * 16)) = widen_e4m3x8(st.w[i][2], st.w[i][3]);
                } else {
                    *(u32x4 *)(to + r * L::kRowBytes + ((piece ^ sw) * 16)) = st.w[i];
                }
            }
        }
        if (E4M3 && wave == scale_wave) ((float *)(lds_s + ((is_v ? L::kRing : 0) + slot) * L::kScale))[lane] = st.scale;
    };
    auto load_k = [&](int t, int page, Staged &st) { load(a.kv.k, a.kv.k_scales, t, page, 0, st); };
    auto load_v = [&](int t, int page, Staged &st) { load(a.kv.v, a.kv.v_scales, t, page, 1, st); };

    f32x16 acc[NR][DT];
    float m[NR], l[NR];
#pragma unroll
    for (int rh = 0; rh < NR; ++rh) {
        m[rh] = kNegInf;
        l[rh] = 0.f;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[rh][dt][e] = 0.f;
    }

    // LDS addresses of this lane's fragments: the rows' places and the lane's part of the chunk; step and D enter by exclusive or
    const uint32_t at_k = (uint32_t)(uintptr_t)(LdsPtr)lds_k + m32 * L::kRowBytes + ((half ^ L::swz_k(m32)) * 16);
    const uint32_t at_s = (uint32_t)(uintptr_t)(LdsPtr)lds_s + half * 16;
    uint32_t at_v[2];       // the two groups of four positions of a step
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const int i16 = lane & 15, r = 8 * p + 4 * half + (i16 >> 2);
        at_v[p] = (uint32_t)(uintptr_t)(LdsPtr)lds_v + r * L::kRowBytes + (((2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ L::swz_v(r)) * 16) + (i16 & 1) * 8;
    }
    // scores of the 32 positions whose keys lie at `off`
    auto scores = [&](uint32_t off, f32x16 (&z)[NR]) {
        const uint32_t kb = at_k + off;
#pragma unroll
        for (int rh = 0; rh < NR; ++rh)
#pragma unroll
            for (int e = 0; e < 16; ++e) z[rh][e] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const bf16x8 k = *(__attribute__((address_space(3))) const bf16x8 *)(uintptr_t)(kb ^ (ks * 32));
#pragma unroll
            for (int rh = 0; rh < NR; ++rh) z[rh] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[rh][ks], z[rh], 0, 0, 0);
        }
    };
    // adds the values, at `off`, of 32 positions
    auto values = [&](uint32_t off, const bf16x8 (&pf)[2][NR]) {
#pragma unroll
        for (int t16 = 0; t16 < 2; ++t16)
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) {
                union {
                    s16x4 part[2];
                    bf16x8 v;
                } f;
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    f.part[p] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (__attribute__((address_space(3))) s16x4 *)(uintptr_t)(((at_v[p] + off) ^ (dt * 64)) + t16 * 16 * L::kRowBytes));
#pragma unroll
                for (int rh = 0; rh < NR; ++rh) acc[rh][dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, pf[t16][rh], acc[rh][dt], 0, 0, 0);
            }
    };

    bf16x8 pf[2][NR];        // probabilities of the step before: [16 positions][rows]
    f32x16 z[NR];            // scores of this step
    bool rare = false;      // values that are not finite were found in a tile that some row does not see whole
    if (tiles > 0) {
        int pg0 = find_pages(0), pg1 = find_pages(1), pg2 = find_pages(2);
        if (tid == 0) *lds_flag = 0;
        // in front of the first step there are no values: zeros with probability zero
        for (int i = tid; i < 32 * L::kRowBytes / 16; i += kManyThreads) ((u32x4 *)(lds_v + 2 * L::kHalf + 32 * L::kRowBytes))[i] = u32x4{0, 0, 0, 0};
        Staged sk, sv;
        load_k(0, pg0, sk);
        load_v(0, pg0, sv);
        store(false, 0, 0, sk);
        store(true, 0, 1, sv);
        load_k(1, pg1, sk);     // (tiles behind the last one read its positions again)
        store(false, 1, 0, sk);
#pragma unroll
        for (int t16 = 0; t16 < 2; ++t16)
#pragma unroll
            for (int rh = 0; rh < NR; ++rh) pf[t16][rh] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        lds_barrier();
        scores(0, z);
        int slot = 0;       // t % 3
#pragma unroll 1
        for (int t = 0; t < tiles; ++t) {
            const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot == 0 ? 2 : slot - 1;     // (t + 1) % 3, (t + 2) % 3 = (t - 1) % 3
            const int pg3 = find_pages(t + 3);
            load_k(t + 2, pg2, sk);
            load_v(t + 1, pg1, sv);
            const int pos0 = lo + t * kManyTile;
            const unsigned long long holes = __ballot(pg0 < 0);       // positions without a page are not seen
            if (holes != 0 || pos0 < blk_lo || pos0 + kManyTile - 1 > blk_hi) {
                // Some row does not see all of this tile's values, and a product of an infinity or a NaN with the probability 0 is a NaN: such
                // values become zeros in LDS, and the rows that see them get them in the end.
                bool bad = false;
#pragma unroll
                for (int i = 0; i < L::kHalf / 16 / kManyThreads; ++i) {
                    u32x4 *w = (u32x4 *)(lds_v + slot * L::kHalf) + i * kManyThreads + tid;
                    u32x4 v = *w;
                    const u32x4 was = v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = only_finite_bf16(v[e]);
                    if (v[0] != was[0] || v[1] != was[1] || v[2] != was[2] || v[3] != was[3]) {
                        *w = v;
                        bad = true;
                    }
                }
                if (E4M3 && tid < kManyTile) {
                    float *sc = (float *)(lds_s + (L::kRing + slot) * L::kScale) + tid;
                    if (!(fabsf(*sc) < __builtin_inff())) {
                        *sc = 0.f;
                        bad = true;
                    }
                }
                if (bad) *lds_flag = 1;
                lds_barrier();
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int p0 = pos0 + u * 32;
                if (E4M3) {     // the keys' scales
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        const f32x4 f = *(__attribute__((address_space(3))) const f32x4 *)(uintptr_t)(at_s + slot * L::kScale + u * 128 + b * 32);
#pragma unroll
                        for (int rh = 0; rh < NR; ++rh)
#pragma unroll
                            for (int e = 0; e < 4; ++e) z[rh][4 * b + e] *= f[e];
                    }
                }
                if (holes != 0 || p0 < all_lo || p0 + 31 > all_hi) {
                    int j0 = p0 + 4 * half;
                    uint32_t hole = (uint32_t)(holes >> (u * 32)) >> (4 * half);
                    asm volatile("" : "+v"(j0), "+v"(hole));        // (keeps the comparisons' operands in this block)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int k = 8 * (e >> 2) + (e & 3);
#pragma unroll
                        for (int rh = 0; rh < NR; ++rh)
                            if (j0 + k < see_lo[rh] || j0 + k > see_hi[rh] || (hole >> k & 1u)) z[rh][e] = kNegInf;
                    }
                }
                // ---- one block without branches: scores of the next step, values of the last one, probabilities of this one
                f32x16 zn[NR];
                scores(u == 0 ? slot * L::kHalf + 32 * L::kRowBytes : slot1 * L::kHalf, zn);
                values(u == 0 ? slot2 * L::kHalf + 32 * L::kRowBytes : slot * L::kHalf, pf);
                float keep[NR];
                bool moved = false;
#pragma unroll
                for (int rh = 0; rh < NR; ++rh) {
                    float mx = z[rh][0];
#pragma unroll
                    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, z[rh][e]);
                    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                    mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
                    const bool up = mx > m[rh] + stale;         // a row goes by its own scores alone
                    const float to = up ? mx : m[rh];
                    keep[rh] = up ? __builtin_amdgcn_exp2f((m[rh] - to) * c2) : 1.f;
                    moved |= up;
                    m[rh] = to;
                    const float mb = to == kNegInf ? 0.f : to * c2;
                    float sum[2] = {0.f, 0.f};
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        z[rh][e] = __builtin_amdgcn_exp2f(fmaf(z[rh][e], c2, -mb));
                        sum[e & 1] += z[rh][e];
                    }
                    l[rh] = fmaf(l[rh], keep[rh], sum[0] + sum[1]);
#pragma unroll
                    for (int t16 = 0; t16 < 2; ++t16) {
                        float p[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) p[e] = z[rh][8 * t16 + e];
                        if (E4M3) {
#pragma unroll
                            for (int b = 0; b < 2; ++b) {
                                const f32x4 f = *(__attribute__((address_space(3))) const f32x4 *)(uintptr_t)(at_s + (L::kRing + slot) * L::kScale + u * 128 + t16 * 64 + b * 32);
#pragma unroll
                                for (int e = 0; e < 4; ++e) p[4 * b + e] *= f[e];
                            }
                        }
                        pf[t16][rh] = pack_bf16x8(p);
                    }
                }
#pragma unroll
                for (int t16 = 0; t16 < 2; ++t16)
#pragma unroll
                    for (int rh = 0; rh < NR; ++rh) asm volatile("" : "+v"(pf[t16][rh]));      // (keeps the exponentials on this side of the branch)
                if (__ballot(moved) != 0) {
#pragma unroll
                    for (int rh = 0; rh < NR; ++rh)
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) acc[rh][dt] *= keep[rh];
                }
#pragma unroll
                for (int rh = 0; rh < NR; ++rh) z[rh] = zn[rh];
            }
            store(false, slot2, 0, sk);     // the ring's third place: nobody reads K(t - 1) or V(t - 2) any more
            store(true, slot1, 1, sv);
            lds_barrier();
            pg0 = pg1;
            pg1 = pg2;
            pg2 = pg3;
            slot = slot1;
        }
        const int last = slot == 0 ? 2 : slot - 1;      // (tiles - 1) % 3
        values(last * L::kHalf + 32 * L::kRowBytes, pf);
        rare = *lds_flag != 0;
    }
    if (rare) {
        // Those values went into no product (0 * inf is NaN in the rows that do not see them): the rows that see them get them here.
#pragma unroll 1
        for (int j = max(lo, any_lo); j < min(hi, any_hi + 1); ++j) {
            const int t0 = lo + ((j - lo) & ~(kManyTile - 1));      // its tile
            const int page = table[j >> shift];
            bool whole = t0 >= blk_lo && t0 + kManyTile - 1 <= blk_hi;
            for (int i = 0; whole && i < kManyTile; i += 8) {       // (a tile with a missing page counts as masked)
                const int other = table[min(max(t0 + i, begin), end - 1) >> shift];
                whole = other >= 0 && other < a.kv.num_pages;
            }
            if (whole || page < 0 || page >= a.kv.num_pages) continue;
            const int64_t at = head_page(page) + (j & ((1 << shift) - 1));
            const float vs = E4M3 ? a.kv.v_scales[at] : 1.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int64_t d = at * D + 32 * dt + 8 * (e >> 2) + 4 * half + (e & 3);
                    const float v = E4M3 ? vs * __builtin_amdgcn_cvt_f32_fp8((int)((const uint8_t *)a.kv.v)[d], 0) : bf16_bits_to_f32(((const uint16_t *)a.kv.v)[d]);
                    const bool bad = !(fabsf(v) < __builtin_inff());
#pragma unroll
                    for (int rh = 0; rh < NR; ++rh)
                        if (bad && j >= see_lo[rh] && j <= see_hi[rh]) acc[rh][dt][e] += v;
                }
        }
    }
#pragma unroll
    for (int rh = 0; rh < NR; ++rh) {
        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l[rh]), __float_as_uint(l[rh]), false, false);
        const float sum = __uint_as_float(both[0]) + __uint_as_float(both[1]);
        const int in_rows = (wave * NR + rh) * 32 + m32;
        if (in_rows >= in_block) continue;
        const int64_t row = row0 + in_rows, qi = row / G;
        const int64_t out_row = (sr.row_lo + qi) * a.q_heads + h * G + (row - qi * G);
        // lane (row n, half) holds D index 32 dt + 8 (e / 4) + 4 half + e % 4
        const float inv = inverse_sum(sum);
        float *po = parts.o + ((int64_t)split * parts.rows + out_row) * D;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                f32x4 o = {acc[rh][dt][4 * b], acc[rh][dt][4 * b + 1], acc[rh][dt][4 * b + 2], acc[rh][dt][4 * b + 3]};
                const int d = 32 * dt + 8 * b + 4 * half;
                if (pieces == 1) store_out4(a, out_row, D, d, o * inv);
                else *(f32x4 *)(po + d) = o;
            }
        if (half == 0) {
            if (pieces == 1) {
                if (a.lse) a.lse[out_row] = (m[rh] * c2 + __builtin_amdgcn_logf(sum)) * kLn2;
            } else {
                parts.ml[((int64_t)split * parts.rows + out_row) * 2] = m[rh] * c2;
                parts.ml[((int64_t)split * parts.rows + out_row) * 2 + 1] = sum;
            }
            if (split == 0 && parts.splits > 0) parts.count[out_row] = pieces;
        }
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
    attention_tile_kernel<D, E4M3><<<dim3((unsigned)grid), dim3(kManyThreads), ManyLayout<D>::kLds, s>>>(a, 16 * p.few_nr, p.tile_chunk, p.tile_blocks, parts);
    return check_hip(hipGetLastError(), "attention_tile_kernel");
}

int launch_attention_tile(const AttnArgs &a, const AttnPlan &p, const AttnParts &parts, hipStream_t s)
{
    const bool e4m3 = a.kv.fmt == QARL_KV_E4M3;
    if (a.kv.head_dim == 128) return e4m3 ? launch_tile_as<128, true>(a, p, parts, s) : launch_tile_as<128, false>(a, p, parts, s);
    return e4m3 ? launch_tile_as<64, true>(a, p, parts, s) : launch_tile_as<64, false>(a, p, parts, s);
}

}  // namespace qarl
