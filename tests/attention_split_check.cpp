// Random calls of the attention, split on the host by the code that the kernels and their launcher run.  Prints the first calls that break a rule and
// returns how many there were.  Built and run by test_attention_split.py.
#include <cmath>
#include <cstdio>
#include <random>
#include <vector>
#include "attention_split.hpp"

using namespace qarl;

static std::mt19937_64 rng;
static int64_t pick(int64_t lo, int64_t hi) { return lo + (int64_t)(rng() % (uint64_t)(hi - lo + 1)); }
static int64_t spread(int64_t lo, int64_t hi)     // evenly over the logarithm
{
    const double u = (double)(rng() >> 11) / 9007199254740992.0;
    return std::min(hi, std::max(lo, (int64_t)std::llround(std::exp(std::log((double)lo) + u * (std::log((double)hi) - std::log((double)lo))))));
}

int main(int argc, char **argv)
{
    const long calls = std::atol(argv[1]);
    long bad = 0;
    for (long c = 0; c < calls; ++c) {
        rng.seed(c + 1);
        AttnArgs a = {};
        a.kv.kv_heads = (int)pick(1, 8);
        const int G = (int)(pick(0, 3) ? pick(1, 16) : pick(1, 128));
        a.q_heads = a.kv.kv_heads * G;
        a.S = (int)spread(1, 60);
        a.max_q_len = (int)(pick(0, 2) ? spread(1, 700) : 1);
        std::vector<int32_t> offsets = {0}, kv;
        for (int s = 0; s < a.S; ++s) {
            // most sequences within the bound, some longer; as many cached positions as queries, more, fewer, more than the bounds and the table allow
            const int n = (int)(pick(0, 9) ? pick(0, a.max_q_len) : pick(0, 3 * a.max_q_len + 300));
            offsets.push_back(offsets.back() + n);
            kv.push_back((int)(pick(0, 5) ? n + spread(1, 6000) - 1 : pick(0, n)));
        }
        a.T = offsets.back();
        if (a.T == 0) continue;
        a.q_offsets = offsets.data();
        a.kv_lens = kv.data();
        a.max_kv_len = (int)spread(1, 9000);
        a.kv.page_shift = (int)pick(3, 7);
        a.table_width = (int)spread(1, 8000 >> a.kv.page_shift);
        a.window = (int)(pick(0, 2) ? spread(1, 6000) : 0);
        const AttnPlan p = attention_plan(a.T, a.q_heads, a.kv.kv_heads, a.S, a.max_q_len, a.max_kv_len, a.window);
        const AttnPlan room = attention_plan(a.T, a.q_heads, a.kv.kv_heads, a.S, a.max_q_len, a.max_kv_len, 0);
        const char *broken = p.splits > room.splits ? "more room with a window than the workspace query names" : nullptr;
        if (p.few_nr && (p.few_chunk % 128 || p.few_chunk > 8192)) broken = "pieces of few rows that the list of pages does not hold";
        int64_t blocks = 0;
        for (int s = 0; s < a.S; ++s) {
            const SeqRange r = seq_range(a, s);
            if (r.n == 0) continue;
            const int64_t rows = (int64_t)r.n * G;
            const bool few = p.few_nr && rows <= 16 * p.few_nr;
            blocks += few ? 0 : (rows + kManyRows - 1) / kManyRows;
            if (over_long(a, r)) {
                if (!p.few_nr && !p.tile) broken = "nobody notes that a sequence is left out";
                continue;
            }
            if (!few && !p.tile) {
                broken = "a sequence that no kernel takes";
                continue;
            }
            const int unit = few ? kFewTile : kManyTile, chunk = few ? p.few_chunk : p.tile_chunk, splits = few ? p.few_splits : p.tile_splits;
            for (int64_t row0 = 0; row0 < rows; row0 += few ? rows : kManyRows) {
                const int64_t last = few ? rows - 1 : std::min(row0 + kManyRows, rows) - 1;
                int begin, end;
                visible_range(a, r, (int)(row0 / G), (int)(last / G), begin, end);
                const Pieces cut = cut_range(begin, end, unit, chunk);
                if (begin >= end && end - cut.base > 0) broken = "tiles of positions that nobody sees";
                if (end > a.max_kv_len || end > (a.table_width << a.kv.page_shift)) broken = "positions past the bounds";
                if (cut.count > splits) broken = "more pieces than are launched";
                if (cut.count > std::max(1, p.splits)) broken = "more pieces than there is room for";
            }
        }
        if (p.tile && blocks > p.tile_blocks) broken = "more row blocks than are launched";
        if (broken && bad++ < 10)
            std::printf("call %ld: %s (T %d, heads %d on %d, S %d, max_q_len %d, max_kv_len %d, table %d pages of %d, window %d)\n", c, broken, a.T, a.q_heads,
                        a.kv.kv_heads, a.S, a.max_q_len, a.max_kv_len, a.table_width, 1 << a.kv.page_shift, a.window);
    }
    std::printf("%ld calls, %ld broken\n", calls, bad);
    return bad != 0;
}
