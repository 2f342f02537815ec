// How a call of the attention over the paged cache is split: which kernel takes a sequence, into how many pieces its cache is cut, and which positions
// a run of its queries sees.  Host and device; tests/test_attention_split.py runs it on the host.
#pragma once
#include "common.hpp"

namespace qarl {

// How a call is split: each kernel takes the sequences whose row count (queries times G) lies on its side of few_rows, and cuts a
// sequence's cache into pieces of `chunk` positions.
struct AttnPlan {
    int few_nr;        // the kernel for few rows: 16 * few_nr rows at a time; 0: not launched
    int few_chunk, few_splits;
    int tile;          // the kernel for many rows is launched
    int tile_chunk, tile_splits, tile_blocks;   // tile_blocks: bound of the row blocks of one cached head
    int splits;        // room for partial results per row (0: none)
};

constexpr int kFewTile = 32;      // positions a wavefront of the few-row kernel takes at a time
constexpr int kManyTile = 64;     // positions of a tile of the many-row kernel
constexpr int kManyWaves = 8, kManyRows = 256;

struct SeqRange {
    int row_lo, n;        // first query row, queries
    int kv;               // cached positions, as the caller gives them: query i stands at kv - n + i
    int cap;              // positions from here on do not exist
};

__host__ __device__ inline SeqRange seq_range(const AttnArgs &a, int s)
{
    SeqRange r;
    const int lo = max(0, min(a.T, a.q_offsets[s])), hi = max(0, min(a.T, a.q_offsets[s + 1]));
    r.row_lo = lo;
    r.n = max(0, hi - lo);
    r.kv = max(0, a.kv_lens[s]);
    const int64_t table = (int64_t)a.table_width << a.kv.page_shift;
    r.cap = (int)min((int64_t)min(r.kv, a.max_kv_len), table);
    return r;
}

// Positions [begin, end) that queries [i0, i1] see between them.  None (a query in front of the first position, a window that starts behind the last one
// there is): 0, 0, so that no tile is made of them; the tiles' reads stay within a range by its first and last position, which then do not exist.
__host__ __device__ inline void visible_range(const AttnArgs &a, const SeqRange &s, int i0, int i1, int &begin, int &end)
{
    const int64_t p0 = (int64_t)s.kv - s.n + i0, p1 = (int64_t)s.kv - s.n + i1;
    const int64_t e = min(p1 + 1, (int64_t)s.cap);
    const int64_t b = a.window > 0 ? max((int64_t)0, p0 - a.window + 1) : 0;
    end = e > b ? (int)e : 0;
    begin = e > b ? (int)b : 0;
}

// What a row sees: positions lo <= j <= hi
__host__ __device__ inline void row_bounds(const AttnArgs &a, const SeqRange &s, int i, int &lo, int &hi)
{
    const int64_t p = (int64_t)s.kv - s.n + i;
    hi = (int)min(p, (int64_t)s.cap - 1);
    lo = a.window > 0 ? (int)max((int64_t)0, p - a.window + 1) : 0;
}

// A sequence of more queries than the call allows for.  The pieces of a window's positions, and with them the room for partial results, go by
// max_q_len: both kernels leave such a sequence out, and the join finds no pieces of its rows.
__host__ __device__ inline bool over_long(const AttnArgs &a, const SeqRange &s) { return s.n > a.max_q_len; }

// Positions [begin, end) in pieces of `chunk`, from the tile of `unit` positions that holds the first one on
struct Pieces {
    int base, count;
};
__host__ __device__ inline Pieces cut_range(int begin, int end, int unit, int chunk)
{
    const int base = begin & ~(unit - 1);
    return Pieces{base, max(1, (end - base + chunk - 1) / chunk)};
}

// Pieces per (sequence, head) so that they fill 256 CUs one to four times, at the least cost for sequences of the longest length: positions, and for
// each piece's start and end as much as `extra` of them take.  (Shorter lengths never give more pieces: the room for partial results relies on it.)
inline int64_t few_pieces(int64_t units, int64_t len, int64_t extra)
{
    int64_t best = 1, times = 1;
    for (int64_t r = 1; r <= 4; ++r) {
        const int64_t n = 256 * r / units;
        if (r == 1 || r * (len + extra * n) * best < times * (len + extra * best) * n) best = n, times = r;
    }
    return best;
}

// Sequences with at most 64 rows per cached head go to the kernel whose wavefronts share a sequence's positions, others to the one whose wavefronts
// share its rows.  Both cut a cache into pieces where there are not enough (sequence, head, row block)s to fill the 256 CUs; partial results cost
// 2 D fp32 per row and piece.
//   Few rows: pieces of 512 positions or more (a single sequence of 18432 with 256 / 384 / 512 at least: 20.7 / 16.2 / 16.0 us).  A CU holds one workgroup, or two
//   whose rings are 64 KiB.
//   From 256 (sequence, head)s on about four pieces per CU at the longest length, for the lengths are not known here: 64 ragged sequences of up to
//   18000, 4 heads, 8 / 32 / 64 rows with one piece 232 / 253 / 327, with four 211 / 232 / 290 (of equal lengths 8000, 32 / 64 rows, the other way:
//   190 / 204 against 207 / 244).  Below that few_pieces(): 16 of 4096, 8 / 64 rows 34 / 46 instead of 40 / 69 with four pieces per CU; 48 of 12000, 64 rows,
//   with 256 / 512 / 768 / 1024 wanted 282 / 300 / 257 / 282 (24 ragged ones of up to 12000, 64 rows, lose: 114 instead of 109).
//   At the border one and four pieces are close, 252 and 256 (sequence, head)s alike: 64 sequences of up to 9000 with one / four, single tokens bf16 211 / 212, e4m3
//   117 / 121, ragged 118 / 115 and 81 / 65; 64 rows 238 / 264, 186 / 208, ragged 167 / 164, 151 / 146; 63 sequences within 3 % of that, e4m3 ragged 82 / 65.
//   Many rows: a workgroup per CU; beyond 128 blocks a cut costs what it fills (1 x 2048 over 16384, 256 blocks: 626 us whole, 658 in two; 512 over 8192, 64
//   blocks: 244 whole, 92 in four, 107 in eight; 4 x 300 over 4000, 160 blocks: 133 whole, 158 in two, 151 in four; 2 x 700 over 12000, 176 blocks: 419
//   whole, 450 in two, 393 in four).
inline AttnPlan attention_plan(int T, int q_heads, int kv_heads, int S, int max_q_len, int max_kv_len, int window)
{
    AttnPlan p = {};
    const int64_t G = q_heads / kv_heads;
    const int64_t most = min((int64_t)max_q_len, (int64_t)T);
    const bool all_few = most * G <= 64;
    const int64_t few_rows = all_few ? most * G : G;         // beside long chunks: single tokens
    p.few_nr = few_rows <= 16 ? 1 : few_rows <= 32 ? 2 : few_rows <= 64 ? 4 : 0;
    // can a sequence be that short, where the others are at most `most` long?
    if (!all_few && T > (int64_t)(S - 1) * most + 16 * p.few_nr / G) p.few_nr = 0;
    p.tile = !all_few;
    int64_t len = max_kv_len > 0 ? max_kv_len : 1;
    if (window > 0) len = min(len, (int64_t)window + most + kManyTile);
    // (the room for partial results goes by n, not by the pieces that the rounded length gives: it must not grow when a window shortens len)
    const auto cut = [len, &p](int64_t n, int64_t unit, int64_t most_len, int &chunk, int &splits) {
        n = max(min(n, (len + 511) / 512), (int64_t)1);
        chunk = (int)min(((len + n - 1) / n + unit - 1) / unit * unit, most_len);
        splits = (int)((len + chunk - 1) / chunk);
        p.splits = max(p.splits, max((int)n, splits));
    };
    if (p.few_nr) {
        const int64_t units = (int64_t)S * kv_heads;
        cut(units >= 256 ? (1024 + units - 1) / units : few_pieces(units, len, p.few_nr == 4 ? 512 : 256), 128, 8192, p.few_chunk, p.few_splits);
    }
    if (p.tile) {
        p.tile_blocks = (int)((T * G + kManyRows - 1) / kManyRows + min((int64_t)S, (int64_t)T));      // a bound
        const bool even = T == (int64_t)S * most;
        const int64_t blocks = kv_heads * (even ? S * ((most * G + kManyRows - 1) / kManyRows) : T * G / kManyRows + S / 2 + 1);
        cut(blocks <= 128 ? 256 / blocks : 1, 64, (int64_t)1 << 30, p.tile_chunk, p.tile_splits);
    }
    if (p.splits <= 1) p.splits = 0;
    return p;
}

}  // namespace qarl
