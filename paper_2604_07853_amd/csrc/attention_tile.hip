// Attention of many query rows per sequence (prompts, chunks of prompts) over the paged cache.
// Bound by what the SIMDs issue, products and softmax together.  A workgroup takes a block of 256 rows of one cached head (rows are (query, head of the
// group)) and runs over the cache in tiles of 64 positions, which its eight wavefronts share through rings of three tiles in LDS.
//
// S^T = K Q^T and O^T = V^T P^T on 32 x 32 x 16 matrix instructions: a wavefront owns 32 rows, two wavefronts share a SIMD.  (64 rows would halve the LDS
// reads, but spill 600 registers beside a second wavefront, and without one move 300 a tile between the two register files.)  Lane (n = lane & 31,
// half = lane >> 5) holds row n's scores at positions 8 (i / 4) + 4 half + i % 4, i = 0 .. 15, of 32 positions: the maximum and the sum of a row are
// in-lane but for one exchange between the halves, and registers 8 t .. 8 t + 7, packed to bf16, are the B operand of step t of the second product as
// they are (contraction order {4 half + 0..3, 8 + 4 half + 0..3} of 16 positions).  V^T in that order lies in LDS: a tile's values are transposed on their way.
//
// A wavefront's own work overlaps: step s (32 positions) computes the scores of step s + 1 and adds the values of step s - 1 on the matrix cores while the
// vector units turn the scores of step s into probabilities; none of the three waits for another.
//
// Measured, 32 query heads on 4 cached ones of 128, calls on end: eight prompts of 2048 bf16 352 us (275 GFLOP, 781 TFLOP/s), e4m3 384 (716), with a window of
// 512 210 (572), head_dim 64 236 (584); 4 x 2048 over 16384 cached positions 2288 us (1021 TFLOP/s); 28 heads on 4, 12 chunks of mixed lengths over an e4m3
// cache 332 us (781 TFLOP/s).  The first ten calls after a pause of 50 ms take 438 us for the prompts and 419 for the chunks; under the profiler 384 and 345.  A
// tile takes 4040-4160 cycles, 2048 of them products; a block 7 us more to start and end.
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
    // Keys: [position][D], chunk c of row r at c ^ swz_k(r), so that the rows that one read touches at the same chunk spread over the banks.
    __device__ static constexpr int swz_k(int r) { return (r / (256 / kRowBytes)) & (kChunks - 1); }
    // Values: transposed, [D][64 positions], the positions of each 16 in the order 0..3, 8..11, 4..7, 12..15, so that a lane's eight of a step are one
    // 16-byte chunk (transposing reads of row-major tiles deliver 182 bytes per ns and CU, 16-byte reads 335); chunk c of row d at c ^ swz_v(d).
    __device__ static constexpr int swz_v(int d) { return (d ^ (d >> 3)) & 7; }
    __device__ static constexpr int at_v(int pos) { return (pos & 0x33) | (pos & 4) << 1 | (pos & 8) >> 1; }
};

template <int D, bool E4M3>
__global__ __launch_bounds__(kManyThreads, 2) void attention_tile_kernel(AttnArgs a, int few_rows, int chunk, int blocks, AttnParts parts)
{
    using L = ManyLayout<D>;
    constexpr int KS = D / 16, DT = D / 32;
    extern __shared__ __align__(128) char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int m32 = lane & 31, half = lane >> 5;
    const int Hkv = a.kv.kv_heads, G = a.q_heads / Hkv;
    // workgroup -> (piece, row block, cached head), heads fastest: workgroup ids go round the 8 XCDs, so an XCD meets few heads and its L2 keeps them;
    // a sequence's later row blocks, which see more of the cache, first
    const unsigned per_split = (unsigned)blocks * (unsigned)Hkv;
    const int split = (int)(blockIdx.x / per_split);
    const unsigned bh = blockIdx.x - (unsigned)split * per_split;
    const int h = (int)(bh % (unsigned)Hkv);
    int block = (int)(bh / (unsigned)Hkv);
    // the sequence of the row block: 64 sequences at a time, one per lane
    int s = -1;
    SeqRange sr;
    for (int s0 = 0; s0 < a.S; s0 += 64) {
        const SeqRange mine = seq_range(a, min(s0 + lane, a.S - 1));
        const int rows = mine.n * G;                    // (below 2^31: checked on the host)
        const int nb = s0 + lane < a.S && rows > few_rows ? (int)((unsigned)(rows + kManyRows - 1) / kManyRows) : 0;
        // blocks in front of this sequence's: of up to 64 sequences those with longer caches come first (a workgroup's time goes by the cache, and a long
        // one that starts last is waited for: 12 sequences of up to 8900 positions 432 -> 368 us), of more sequences those with lower numbers
        int before = 0;
        if (a.S <= 64 && __ballot(mine.kv != __builtin_amdgcn_readfirstlane(mine.kv)) != 0) {
            for (int j = 0; j < a.S; ++j) {
                const int kv = __builtin_amdgcn_readlane(mine.kv, j), n = __builtin_amdgcn_readlane(nb, j);
                before += kv > mine.kv || (kv == mine.kv && j < lane) ? n : 0;
            }
        } else {
            int incl = nb;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int up = __shfl_up(incl, o, 64);
                if (lane >= o) incl += up;
            }
            before = incl - nb;
        }
        const unsigned long long hit = __ballot(block >= before && block < before + nb);
        if (hit) {
            const int src = __ffsll((long long)hit) - 1;
            s = s0 + src;
            block = __builtin_amdgcn_readlane(nb, src) - 1 - (block - __builtin_amdgcn_readlane(before, src));
            sr.row_lo = __builtin_amdgcn_readlane(mine.row_lo, src);
            sr.n = __builtin_amdgcn_readlane(mine.n, src);
            sr.kv = __builtin_amdgcn_readlane(mine.kv, src);
            sr.cap = __builtin_amdgcn_readlane(mine.cap, src);
            break;
        }
        block -= __builtin_amdgcn_readlane(before + nb, 63);
    }
    if (s < 0) return;                                  // the grid is a bound
    const int row0 = block * kManyRows, in_block = min(kManyRows, sr.n * G - row0);
    const int i_first = (int)((unsigned)row0 / (unsigned)G), i_last = (int)((unsigned)(row0 + in_block - 1) / (unsigned)G);
    if (over_long(a, sr)) {
        if (split == 0 && parts.splits > 0) {
            for (int r = row0 + tid; r < row0 + in_block; r += kManyThreads) {
                const int i = (int)((unsigned)r / (unsigned)G);
                parts.count[(int64_t)(sr.row_lo + i) * a.q_heads + (h * G + r - i * G)] = 0;
            }
        }
        return;
    }
    int begin, end;
    visible_range(a, sr, i_first, i_last, begin, end);
    const auto [base, pieces] = cut_range(begin, end, kManyTile, chunk);
    if (split >= pieces) return;
    const int lo = base + split * chunk, hi = min(end, lo + chunk);
    const int tiles = (hi - lo + kManyTile - 1) / kManyTile;
    const int shift = a.kv.page_shift;
    const int32_t *table = a.table + (int64_t)s * a.table_stride;

    // this lane's row: queries as B operand, bounds of what it sees
    bf16x8 qf[KS];
    int see_lo, see_hi;
    const int in_rows = wave * 32 + m32;
    const int row = row0 + (in_rows < in_block ? in_rows : 0), qi = (int)((unsigned)row / (unsigned)G);
    const int64_t out_row = (int64_t)(sr.row_lo + qi) * a.q_heads + (h * G + row - qi * G);
    {
        row_bounds(a, sr, qi, see_lo, see_hi);
        if (in_rows >= in_block || see_hi < see_lo) {
            see_lo = 0x40000000;
            see_hi = see_lo;
        }
        const uint16_t *qp = (const uint16_t *)a.q + (int64_t)(sr.row_lo + qi) * a.q_token_stride + (int64_t)(h * G + row - qi * G) * a.q_head_stride;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            u32x4 w = *(const u32x4 *)(qp + 16 * ks + 8 * half);
            if (a.scale < 0.f) w ^= 0x80008000u;        // scores go by the scale's size: the running maximum wants it positive
            if (a.scale == 0.f) {                       // zeros, but for infinities and NaN
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] ^= only_finite_bf16(w[e]);
            }
            qf[ks] = __builtin_bit_cast(bf16x8, w);
        }
    }
    // (scale 0: the scores are zeros, infinities or NaN already, and 0 times the maximum's start -inf would be a NaN; the lag has to be finite for the same start)
    const float c2 = a.scale == 0.f ? 1.f : fabsf(a.scale) * kLog2e, stale = fminf(kStale / c2, 3e38f);
    // positions [all_lo, all_hi] are seen by all rows of the wavefront, [any_lo, any_hi] by one at least (a wavefront without rows: none)
    int all_lo, all_hi, any_lo, any_hi;
    {
        const int w_first = (int)((unsigned)(row0 + wave * 32) / (unsigned)G), w_last = (int)((unsigned)(row0 + min(in_block - 1, wave * 32 + 31)) / (unsigned)G);
        row_bounds(a, sr, w_first, any_lo, all_hi);
        row_bounds(a, sr, w_last, all_lo, any_hi);
        if (wave * 32 >= in_block) any_hi = -64;
        any_lo = __builtin_amdgcn_readfirstlane(any_lo);
        any_hi = max(__builtin_amdgcn_readfirstlane(any_hi), -64);
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
        const int page = table[(unsigned)clamp_pos(lo + min(t, tiles - 1) * kManyTile + lane, begin, end - 1) >> shift];
        return (unsigned)page < (unsigned)a.kv.num_pages ? page : -1;
    };
    // positions outside [begin, end), which may hold anything, are not read: the nearest one inside is, again
    auto in_page = [&](int pos) -> int { return clamp_pos(pos, begin, end - 1) & ((1 << shift) - 1); };
    auto head_page = [&](int page) -> int64_t { return ((int64_t)max(page, 0) * Hkv + h) << shift; };
    // ---- a tile's way from the cache through registers into LDS.
    // Keys: a thread moves 16-byte pieces, kStep positions apart; the 4, 8 or 16 neighbouring positions of a wavefront's load lie in one page, or each
    // eight of them do.  Values: a thread takes eight of D at two neighbouring positions and stores them as eight pairs; a wavefront's positions are 8 or 16.
    constexpr int kPieces = D * (E4M3 ? 1 : 2) / 16;                   // 16-byte pieces of a row of the cache
    constexpr int kPer = 64 / kPieces, kLoads = kManyTile * kPieces > kManyThreads ? kManyTile * kPieces / kManyThreads : 1, kStep = kManyWaves * kPer;
    constexpr bool kHalfBusy = kManyTile * kPieces < kManyThreads;     // (e4m3, D = 64: four of the eight wavefronts)
    constexpr int kEights = D / 8, kVPer = 2 * 64 / kEights;           // positions of a wavefront's load of values
    const int k_row = wave * kPer + lane / kPieces, k_piece = lane % kPieces;
    const int v_row = wave * kVPer + lane / kEights * 2, v_d = lane % kEights * 8;
    struct Staged {
        u32x4 k[kLoads], v[2];
        float scale;
    };
    auto row_page = [&](int page, int first, int per) -> int {        // the page of this lane's row of a wavefront's `per` positions from `first` on
        const int pg = __builtin_amdgcn_readlane(page, first & (kManyTile - 1));
        const int second = __builtin_amdgcn_readlane(page, (first + 8) & (kManyTile - 1));
        return per > 8 && lane >= 32 ? second : pg;
    };
    auto load = [&](int tk, int page_k, int tv, int page_v, Staged &st) {
        if (!kHalfBusy || wave < kManyWaves / 2) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const uint32_t in = (uint32_t)in_page(lo + tk * kManyTile + k_row + i * kStep) * (uint32_t)(kPieces * 16) + (uint32_t)(k_piece * 16);
                st.k[i] = *(const u32x4 *)((const char *)a.kv.k + head_page(row_page(page_k, i * kStep + wave * kPer, kPer)) * (kPieces * 16) + in);
            }
        }
        if (D == 128 || wave < kManyWaves / 2) {
            const char *first = (const char *)a.kv.v + head_page(row_page(page_v, wave * kVPer, kVPer)) * (kPieces * 16);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t in = (uint32_t)in_page(lo + tv * kManyTile + v_row + i) * (uint32_t)(kPieces * 16) + (uint32_t)(v_d * (E4M3 ? 1 : 2));
                if (E4M3) {
                    const u32x2 w = *(const u32x2 *)(first + in);
                    st.v[i][0] = w[0];
                    st.v[i][1] = w[1];
                } else {
                    st.v[i] = *(const u32x4 *)(first + in);
                }
            }
        }
        if (E4M3 && wave == 0) st.scale = a.kv.k_scales[head_page(page_k) + in_page(lo + tk * kManyTile + lane)];
        if (E4M3 && wave == 1) st.scale = a.kv.v_scales[head_page(page_v) + in_page(lo + tv * kManyTile + lane)];
    };
    auto store_k = [&](int slot, const Staged &st) {
        if (!kHalfBusy || wave < kManyWaves / 2) {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int r = k_row + i * kStep;
                char *to = lds_k + slot * L::kHalf + r * L::kRowBytes;
                if (E4M3) {
                    *(bf16x8 *)(to + (((2 * k_piece) ^ L::swz_k(r)) * 16)) = widen_e4m3x8(st.k[i][0], st.k[i][1]);
                    *(bf16x8 *)(to + (((2 * k_piece + 1) ^ L::swz_k(r)) * 16)) = widen_e4m3x8(st.k[i][2], st.k[i][3]);
                } else {
                    *(u32x4 *)(to + ((k_piece ^ L::swz_k(r)) * 16)) = st.k[i];
                }
            }
        }
        if (E4M3 && wave == 0) ((float *)(lds_s + slot * L::kScale))[lane] = st.scale;
    };
    // Where some row does not see all of a tile's values (`partly`): the product of an infinity or a NaN with the probability 0 is a NaN.  Such values
    // become zeros, and the rows that see them get them in the end.
    auto store_v = [&](int slot, bool partly, Staged &st) {
        bool bad = false;
        if (D == 128 || wave < kManyWaves / 2) {
            u32x4 w[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = E4M3 ? __builtin_bit_cast(u32x4, widen_e4m3x8(st.v[i][0], st.v[i][1])) : st.v[i];
            if (partly) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t fine = only_finite_bf16(w[i >> 2][i & 3]);
                    bad |= fine != w[i >> 2][i & 3];
                    w[i >> 2][i & 3] = fine;
                }
            }
            const int p = L::at_v(v_row);
            char *to = lds_v + slot * L::kHalf + v_d * 128 + (p & 7) * 2;
#pragma unroll
            for (int i = 0; i < 8; ++i)     // rows d = v_d + i: swz_v(d) = i ^ (v_d / 8)
                *(uint32_t *)(to + i * 128 + (((p >> 3) ^ i ^ (v_d >> 3)) & 7) * 16) =
                    __builtin_amdgcn_perm(w[1][i >> 1], w[0][i >> 1], i & 1 ? 0x07060302u : 0x05040100u);
        }
        if (E4M3 && wave == 1) {
            if (partly && !(fabsf(st.scale) < __builtin_inff())) {
                st.scale = 0.f;
                bad = true;
            }
            ((float *)(lds_s + (L::kRing + slot) * L::kScale))[lane] = st.scale;
        }
        if (partly && bad) *lds_flag = 1;
    };
    auto partly = [&](int t, int page) -> bool {        // is tile t masked for some row of the block?
        const int p0 = lo + t * kManyTile;
        return p0 < blk_lo || p0 + kManyTile - 1 > blk_hi || __ballot(page < 0) != 0;
    };

    f32x16 acc[DT];
    float m = kNegInf, l = 0.f;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[dt][e] = 0.f;

    // LDS addresses of this lane's fragments: the rows' places and the lane's part of the chunk; step and D enter by exclusive or
    const uint32_t at_k = (uint32_t)(uintptr_t)(LdsPtr)lds_k + m32 * L::kRowBytes + ((half ^ L::swz_k(m32)) * 16);
    const uint32_t at_s = (uint32_t)(uintptr_t)(LdsPtr)lds_s + half * 16;
    const uint32_t at_v = (uint32_t)(uintptr_t)(LdsPtr)lds_v + m32 * 128 + ((half ^ L::swz_v(m32)) * 16);
    auto k_frag = [&](uint32_t kb, int ks) -> bf16x8 { return *(__attribute__((address_space(3))) const bf16x8 *)(uintptr_t)(kb ^ (ks * 32)); };
    // step i / DT of the 32 positions, 32 of D (rows 32 dt + m32: swz_v differs by 4 in every second 32)
    auto v_frag = [&](uint32_t vb, int i) -> bf16x8 {
        const int t16 = i / DT, dt = i % DT;
        return *(__attribute__((address_space(3))) const bf16x8 *)(uintptr_t)((vb ^ (t16 * 32 + (dt & 1) * 64)) + dt * 32 * 128);
    };
    auto pack2 = [&](float x, float y, const f32x4 &f, int e) -> uint32_t {      // probabilities e and e + 1 (e4m3: times their values' scales)
        return E4M3 ? pack2_bf16(x * f[e & 3], y * f[(e + 1) & 3]) : pack2_bf16(x, y);
    };
    f32x16 zero;
#pragma unroll
    for (int e = 0; e < 16; ++e) zero[e] = 0.f;

    uint32_t pw[8];         // probabilities of the step before, packed: words 0..3 the first 16 positions, 4..7 the others
    f32x16 z;               // scores of this step
    auto probs = [&](int t16) -> bf16x8 { return __builtin_bit_cast(bf16x8, u32x4{pw[4 * t16], pw[4 * t16 + 1], pw[4 * t16 + 2], pw[4 * t16 + 3]}); };
    bool rare = false;      // values that are not finite were found in a tile that some row does not see whole
    if (tiles > 0) {
        int pg0 = find_pages(0), pg1 = find_pages(1), pg2 = find_pages(2);
        if (tid == 0) *lds_flag = 0;
        // in front of the first step there are no values: zeros with probability zero
        for (int i = tid; i < L::kHalf / 16; i += kManyThreads) ((u32x4 *)(lds_v + 2 * L::kHalf))[i] = u32x4{0, 0, 0, 0};
        Staged st, st1;
        load(0, pg0, 0, pg0, st);
        load(1, pg1, 0, pg0, st1);      // (tiles behind the last one read its positions again)
        store_k(0, st);
        lds_barrier();                  // (the flag is written before it can be set)
        store_v(0, partly(0, pg0), st);
        store_k(1, st1);
#pragma unroll
        for (int i = 0; i < 8; ++i) pw[i] = 0;
        lds_barrier();
        z = zero;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_frag(at_k, ks), qf[ks], z, 0, 0, 0);
        int slot = 0;       // t % 3
        // A tile's requests, and what becomes of them behind its products
        int pg3;
        auto request = [&](int t) {
            pg3 = find_pages(t + 3);
            load(t + 2, pg2, t + 1, pg1, st);
        };
        auto pass_on = [&](int t) {
            const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot == 0 ? 2 : slot - 1;
            store_k(slot2, st);     // the ring's third place: nobody reads K(t - 1) or V(t - 2) any more
            store_v(slot1, t + 1 < tiles && partly(t + 1, pg1), st);
            lds_barrier();
            pg0 = pg1;
            pg1 = pg2;
            pg2 = pg3;
            slot = slot1;
        };
        // Tiles [first, behind) hold something that a row of this wavefront sees, in them or in the half tile in front (whose values are still to be
        // added); of the others it only does its share of the moving, which leaves the SIMD to the other wavefront.  (64 sequences of 9 queries over 8000
        // positions, 3 of 8 wavefronts with rows: 307 -> 206 us; eight prompts of 2048, nothing to leave out: the same.  Loops of their own, for a branch
        // around the products in one loop costs 1 %, or 105 spilled registers.)
        const int first = max(0, (any_lo - 32 - lo) >> 6), behind = max(0, min(tiles, ((any_hi + 32 - lo) >> 6) + 1));
        int t = 0;
#pragma unroll 1
        for (; t < min(first, tiles); ++t) {
            request(t);
            pass_on(t);
        }
#pragma unroll 1
        for (; t < behind; ++t) {
            const int slot1 = slot == 2 ? 0 : slot + 1, slot2 = slot == 0 ? 2 : slot - 1;     // (t + 1) % 3, (t + 2) % 3 = (t - 1) % 3
            request(t);
            const int pos0 = lo + t * kManyTile;
            const unsigned long long holes = __ballot(pg0 < 0);       // positions without a page are not seen
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int p0 = pos0 + u * 32;
                // ---- Scores of the next step and values of the last one on the matrix cores, probabilities of this one on the vector units: kSlots
                // products, each with its share of the softmax and the read of the fragment four products on.  (The fences keep it so: left to itself
                // the compiler puts the products side by side, and matrix cores and vector units take turns: 386 us for eight prompts of 2048.)
                constexpr int kSlots = KS + 2 * DT, kEach = 16 / kSlots, kAhead = 4;
                const uint32_t kb = at_k + (u == 0 ? slot * L::kHalf + 32 * L::kRowBytes : slot1 * L::kHalf);
                const uint32_t vb = (at_v + (u == 0 ? slot2 : slot) * L::kHalf) ^ ((1 - u) * 64);
                bf16x8 frag[kSlots];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) frag[i] = i & 1 ? v_frag(vb, i >> 1) : k_frag(kb, i >> 1);
                f32x4 vs[4];
                if (E4M3) {
#pragma unroll
                    for (int b = 0; b < 4; ++b) {
                        vs[b] = *(__attribute__((address_space(3))) const f32x4 *)(uintptr_t)(at_s + (L::kRing + slot) * L::kScale + u * 128 + b * 32);
                        const f32x4 f = *(__attribute__((address_space(3))) const f32x4 *)(uintptr_t)(at_s + slot * L::kScale + u * 128 + b * 32);
#pragma unroll
                        for (int e = 0; e < 4; ++e) z[4 * b + e] *= f[e];
                    }
                }
                if (holes != 0 || p0 < all_lo || p0 + 31 > all_hi) {
                    uint32_t j0 = (uint32_t)(p0 + 4 * half - see_lo), span = (uint32_t)(see_hi - see_lo);
                    asm volatile("" : "+v"(j0), "+v"(span));        // (keeps the comparisons' operands in this block)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (j0 + (uint32_t)(8 * (e >> 2) + (e & 3)) > span) z[e] = kNegInf;
                    if (holes != 0) {
                        const uint32_t hole = (uint32_t)(holes >> (u * 32)) >> (4 * half);
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (hole >> (8 * (e >> 2) + (e & 3)) & 1u) z[e] = kNegInf;
                    }
                }
                float mx = z[0];
#pragma unroll
                for (int e = 1; e < 16; ++e) mx = fmaxf(mx, z[e]);
                const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
                mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
                const bool up = mx > m + stale;         // a row goes by its own scores alone
                const float to = up ? mx : m;
                const float keep = up ? __builtin_amdgcn_exp2f((m - to) * c2) : 1.f;
                m = to;
                const float mb = to == kNegInf ? 0.f : to * c2;
                f32x16 zn = zero;
                uint32_t pn[8];
                float p[16], sum[2] = {0.f, 0.f};
                __builtin_amdgcn_sched_barrier(0);
                __builtin_amdgcn_s_setprio(1);      // 2 % over even terms: a wavefront that feeds the matrix cores goes first
#pragma unroll
                for (int i = 0; i < kSlots; ++i) {
                    if (i + kAhead < kSlots) frag[i + kAhead] = i & 1 ? v_frag(vb, (i + kAhead) >> 1) : k_frag(kb, (i + kAhead) >> 1);
                    if (i & 1) acc[(i >> 1) % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i], probs((i >> 1) / DT), acc[(i >> 1) % DT], 0, 0, 0);
                    else zn = __builtin_amdgcn_mfma_f32_32x32x16_bf16(frag[i], qf[i >> 1], zn, 0, 0, 0);
#pragma unroll
                    for (int x = 0; x < kEach; ++x) {
                        const int e = i * kEach + x;
                        p[e] = __builtin_amdgcn_exp2f(fmaf(z[e], c2, -mb));
                        if (e > 0) sum[(e - 1) & 1] += p[e - 1];
                        if ((e & 1) == 1 && e > 1) {
                            pn[(e >> 1) - 1] = pack2(p[e - 3], p[e - 2], vs[(e - 3) >> 2], e - 3);
                            asm volatile("" : "+v"(pn[(e >> 1) - 1]));
                        }
                        asm volatile("" : "+v"(p[e]), "+v"(sum[(e - 1) & 1]));       // (here, and not where they are used)
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_s_setprio(0);
                pn[7] = pack2(p[14], p[15], vs[3], 14);
                asm volatile("" : "+v"(pn[7]));
                l = fmaf(l, keep, sum[0] + (sum[1] + p[15]));
#pragma unroll
                for (int i = 0; i < 8; ++i) pw[i] = pn[i];
                if (__ballot(up) != 0) {
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) acc[dt] *= keep;
                }
                z = zn;
            }
            pass_on(t);
        }
#pragma unroll 1
        for (; t < tiles; ++t) {
            request(t);
            pass_on(t);
        }
        const int last = slot == 0 ? 2 : slot - 1;      // (tiles - 1) % 3
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i)
            acc[i % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_frag((at_v + last * L::kHalf) ^ 64, i), probs(i / DT), acc[i % DT], 0, 0, 0);
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
                    if (bad && j >= see_lo && j <= see_hi) acc[dt][e] += v;
                }
        }
    }
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    const float sum = __uint_as_float(both[0]) + __uint_as_float(both[1]);
    // lane (row n, half) holds D index 32 dt + 8 (e / 4) + 4 half + e % 4; bf16: the halves exchange what they have of every second eight, 16 bytes a store
    const float inv = inverse_sum(sum);
    const bool live = in_rows < in_block;
    float *po = parts.o + ((int64_t)split * parts.rows + out_row) * D;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        if (pieces == 1 && !a.out_f32) {
#pragma unroll
            for (int b = 0; b < 4; b += 2) {
                uint32_t w[2][2];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
                        w[x][y] = pack2_bf16(acc[dt][4 * (b + x) + 2 * y] * inv, acc[dt][4 * (b + x) + 2 * y + 1] * inv);
                const auto lo2 = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false), hi2 = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
                if (live) *(u32x4 *)((uint16_t *)a.out + out_row * D + 32 * dt + 8 * (b + half)) = u32x4{lo2[0], hi2[0], lo2[1], hi2[1]};
            }
        } else if (live) {
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const f32x4 o = {acc[dt][4 * b], acc[dt][4 * b + 1], acc[dt][4 * b + 2], acc[dt][4 * b + 3]};
                const int d = 32 * dt + 8 * b + 4 * half;
                if (pieces == 1) store_out4(a, out_row, D, d, o * inv);
                else *(f32x4 *)(po + d) = o;
            }
        }
    }
    if (!live) return;
    if (half == 0) {
        if (pieces == 1) {
            if (a.lse) a.lse[out_row] = (m * c2 + __builtin_amdgcn_logf(sum)) * kLn2;
        } else {
            parts.ml[((int64_t)split * parts.rows + out_row) * 2] = m * c2;
            parts.ml[((int64_t)split * parts.rows + out_row) * 2 + 1] = sum;
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
