// The next token of each row of logits, by temperature, top-k, top-p, min-p and one given random number.
//
// Tokens stand in the order of their logits, equal ones by index; token i weighs w_i = e^((z_i - m) / t), m the largest logit.  All three truncations leave a
// beginning of that order, so all that is asked of a row are places in it: the first k tokens, the shortest beginning that holds p of their weight,
// the tokens of weight min_p and more, and the token at which the kept weights reach u times their sum.  A place is found without sorting: by the counts
// and weights of 4096 bins of the order, then of 4096 parts of the bin that it lies in, until that is a single value.
//
// Sums decide between tokens, and a sum that is off by one part in 10^7 takes another token in one of a thousand rows of a wide distribution.  Weights
// are therefore computed in 64 bits and summed as integers, in units of 2^-43: whatever the order of the additions, a row's token is the same.
//
// 16-bit logits have few values: 4096 bins hold those of size 2^-9 to 2^7 one by one, so that a count says all of a bin, weights are computed once a value
// and not once a token, and a place in the order is a bin and a number.  32-bit logits are put into the same bins by their upper halves: these get weights beside
// their counts, and the tokens of a bin that a place lies in are gathered and sorted.  Rows whose other values matter take a general way, which asks for nothing.
//
// A row is read from memory once, and once more in part to find its token.  What bounds it: 16-bit rows of 151936, 256 of them (78 MB): 27.3 us, of which counting
// 17.5 (4.4 TB/s, 1024 threads a CU that wait for the LDS), the choice 4 to 5 (some 200 instructions a wavefront between ten barriers), the token's search 3; with top-k
// and top-k 50, top-p 28.8.  One workgroup a CU: nothing is read while a row is chosen, so 512 rows take 52.4 and 1024 103 (3.0 TB/s).  Longer rows, in parts: 256 of
// 201088 36.4 and 256000 41.2, 1024 of 256000 165.  One row of 151936, in parts: 17.4 and 19.0.  32-bit rows are read three times, for the largest, for the weights and for
// the tokens of the bins that places lie in, and those from memory where they are many: 256 of 151936 113 and 112 us for 467 MB read (4.1 TB/s; the vector units are
// busy 64 % of it), 1024 429 and 440; with top-p alone a fourth time, 140.  37 of 32003 27.0 and 31.9 us: few CUs, a chain of passages.  A place among more than 1024 tokens
// of one upper half costs another passage (3 rows of 2^20 141 us, by the general way 908).  The general way reads a row for each bin and each refinement of each
// place: 256 rows of 151936 with logits past 128 230 us in 16 bits, 250 to 320 in 32; of a thousandth's spread, whose values are all small, 530 to 730 and 640 to 880.
// (In a captured graph.)
#include <stddef.h>

#include <type_traits>

#include "common.hpp"

namespace qarl {

constexpr int kRowThreads = 1024, kRowWaves = kRowThreads / 64, kBins = 4096, kOwn = kBins / kRowThreads;
constexpr float kWindow = 40.f;     // in units of t: what lies further below the maximum shares the last bin (all of it weighs less than 1e-12)
constexpr double kUnit = 8796093022208.0;   // 2^43

// Ascending keys in descending order of the values (-0 and +0 are equal)
__device__ __forceinline__ uint32_t order_key(float z)
{
    const uint32_t u = __float_as_uint(z + 0.f);
    return u ^ (~(uint32_t)((int32_t)u >> 31) & 0x7fffffffu);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float(k ^ (~(uint32_t)((int32_t)k >> 31) & 0x7fffffffu)); }

// A row's elements in 16-byte pieces from the aligned address in front of it on.  (A piece that holds one of the row's bytes lies in one page of memory:
// what is read beside the row is not used.)
template <bool F32>
struct Row {
    static constexpr int kPer = F32 ? 4 : 8;
    const u32x4 *base;
    int off, V, pieces;
    __device__ __forceinline__ Row(const void *logits, int64_t stride, int row, int V_) : V(V_)
    {
        const uintptr_t p = (uintptr_t)logits + (uintptr_t)(row * stride * (F32 ? 4 : 2));
        base = (const u32x4 *)(p & ~(uintptr_t)15);
        off = (int)(p & 15) / (F32 ? 4 : 2);
        pieces = (off + V + kPer - 1) / kPer;
    }
    // f(index, value) of this thread's elements of piece i
    template <typename Fn>
    __device__ __forceinline__ void piece(int i, Fn f) const { elements(i, base[i], f); }
    template <typename Fn>
    __device__ __forceinline__ void elements(int i, u32x4 w, Fn f) const
    {
        const int first = i * kPer - off;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float z = F32 ? __uint_as_float(w[e & 3]) : __uint_as_float(e & 1 ? w[(e >> 1) & 3] & 0xffff0000u : w[(e >> 1) & 3] << 16);
            if ((unsigned)(first + e) < (unsigned)V) f(first + e, z);
        }
    }
    // ... of pieces [from, to), the workgroup together
    template <typename Fn>
    __device__ __forceinline__ void span(int from, int to, Fn f) const
    {
        constexpr int kAhead = 4;       // pieces requested at once
        for (int i = from + (int)threadIdx.x; i < to; i += kAhead * kRowThreads) {
            u32x4 w[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (i + j * kRowThreads < to) w[j] = base[i + j * kRowThreads];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (i + j * kRowThreads < to) elements(i + j * kRowThreads, w[j], f);
        }
    }
    template <typename Fn>
    __device__ __forceinline__ void all(Fn f) const { span(0, pieces, f); }
};

// (2^52 added: the sum's last bit is a unit)
__device__ __forceinline__ unsigned long long weight_units(double w) { return (unsigned long long)__double_as_longlong(w * kUnit + 4503599627370496.0) & 0xfffffffffffffull; }

// e^y for y <= 0 in units of 2^-43, rounded to nearest even; `w`: e^y itself.  y = k ln 2 + r, |r| <= ln 2 / 2: the power series of e^r up to r^12 is within 1e-16
__device__ __forceinline__ unsigned long long weight_of(double y, double &w)
{
    if (!(y > -800.0)) {
        w = 0.0;
        return 0;
    }
    const double k = rint(y * 1.4426950408889634);
    const double r = fma(-k, 1.9082149292705877e-10, fma(-k, 0.6931471803691238, y));       // ln 2 in two parts: the first has 33 bits
    double p = 1.0 / 479001600.0;
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    w = ldexp(p, (int)k);
    return weight_units(w);
}

struct Bins {
    uint32_t count[kBins];
    unsigned long long mass[kBins];
};

// A place in the order: a value, the tokens and the weight in front of its first token, how many tokens have it and what one of them weighs
struct Place {
    uint32_t key;
    uint32_t before, equal;
    unsigned long long mass, each;
    bool there;
};

struct RowLds {
    Bins first, part;
    unsigned long long wave_mass[kRowWaves];
    uint32_t wave_count[kRowWaves];
    uint32_t found, lo, hi, flags;
    uint32_t at_count, at_size;
    unsigned long long at_mass;
};

template <bool F32>
struct RowSampler {
    Row<F32> row;
    RowLds &s;
    float m, bin_scale;
    double inv_t;
    uint32_t tokens;                    // of the row, without those of weight zero by -inf
    unsigned long long whole;           // their weight

    __device__ __forceinline__ unsigned long long weight(float z) const
    {
        double w;
        return weight_of(((double)z - (double)m) * inv_t, w);
    }
    __device__ __forceinline__ int bin(float z) const { return (int)fminf((m - z) * bin_scale, (float)(kBins - 1)); }

    __device__ __forceinline__ static void clear(Bins &b)
    {
        for (int i = threadIdx.x; i < kBins; i += kRowThreads) {
            b.count[i] = 0;
            b.mass[i] = 0;
        }
    }

    // The first bin at which `pass(tokens up to its end, weight up to its end)` holds, into s.found (kBins: none), s.at_*
    template <typename Fn>
    __device__ __forceinline__ void search(const Bins &b, uint32_t count0, unsigned long long mass0, Fn pass)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        __syncthreads();        // (what the search before found has been read)
        uint32_t c[kOwn], csum = 0;
        unsigned long long w[kOwn], wsum = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            c[i] = b.count[threadIdx.x * kOwn + i];
            w[i] = b.mass[threadIdx.x * kOwn + i];
            csum += c[i];
            wsum += w[i];
        }
        uint32_t ci = csum;
        unsigned long long wi = wsum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t cu = __shfl_up(ci, o, 64);
            const unsigned long long wu = __shfl_up(wi, o, 64);
            if (lane >= o) {
                ci += cu;
                wi += wu;
            }
        }
        if (lane == 63) {
            s.wave_count[wave] = ci;
            s.wave_mass[wave] = wi;
        }
        if (threadIdx.x == 0) s.found = kBins;
        __syncthreads();
        uint32_t cb = count0 + ci - csum;
        unsigned long long wb = mass0 + wi - wsum;
        for (int i = 0; i < wave; ++i) {
            cb += s.wave_count[i];
            wb += s.wave_mass[i];
        }
        int mine = kBins;
        uint32_t ca = 0, size = 0;
        unsigned long long wa = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            if (mine == kBins && c[i] && pass(cb + c[i], wb + w[i])) {
                mine = threadIdx.x * kOwn + i;
                ca = cb;
                wa = wb;
                size = c[i];
            }
            cb += c[i];
            wb += w[i];
        }
        if (mine < kBins) atomicMin(&s.found, (uint32_t)mine);
        __syncthreads();
        if (mine < kBins && s.found == (uint32_t)mine) {
            s.at_count = ca;
            s.at_mass = wa;
            s.at_size = size;
        }
        __syncthreads();
    }

    template <typename Fn>
    __device__ __forceinline__ Place find(Fn pass)
    {
        search(s.first, 0, 0, pass);
        const uint32_t at = s.found;
        if (at == kBins) return Place{0, 0, 0, 0, 0, false};
        // the bin's values
        if (threadIdx.x == 0) {
            s.lo = 0xffffffffu;
            s.hi = 0;
        }
        __syncthreads();
        uint32_t lo = 0xffffffffu, hi = 0;
        row.all([&](int, float z) {
            if (z > -__builtin_inff() && (uint32_t)bin(z) == at) {
                const uint32_t k = order_key(z);
                lo = min(lo, k);
                hi = max(hi, k);
            }
        });
        if (lo <= hi) {
            atomicMin(&s.lo, lo);
            atomicMax(&s.hi, hi);
        }
        __syncthreads();
        lo = s.lo;
        hi = s.hi;
        while (lo < hi) {
            int shift = 0;
            while (((hi - lo) >> shift) >= (uint32_t)kBins) ++shift;
            const uint32_t c0 = s.at_count;
            const unsigned long long w0 = s.at_mass;
            clear(s.part);
            __syncthreads();
            row.all([&](int, float z) {
                const uint32_t k = order_key(z);
                if (k >= lo && k <= hi) {
                    atomicAdd(&s.part.count[(k - lo) >> shift], 1u);
                    atomicAdd(&s.part.mass[(k - lo) >> shift], weight(z));
                }
            });
            __syncthreads();
            search(s.part, c0, w0, pass);
            const uint32_t j = s.found;     // there is one: the bin's end passes
            lo += j << shift;
            hi = min(hi, lo + ((1u << shift) - 1u));
        }
        return Place{lo, s.at_count, s.at_size, s.at_mass, weight(key_value(lo)), true};
    }
};

// What is asked of a row
struct RowAsk {
    float t, top_p, min_p, u;
    int k;
    bool greedy;
};
__device__ __forceinline__ RowAsk row_ask(const SampleArgs &a, int r)
{
    RowAsk x;
    x.t = a.temperature ? a.temperature[r] : 1.f;
    x.greedy = x.t == 0.f;
    if (x.greedy) x.t = 1.f;
    x.k = x.greedy ? 1 : a.top_k ? a.top_k[r] : 0;
    x.top_p = a.top_p ? a.top_p[r] : 1.f;
    x.min_p = a.min_p ? a.min_p[r] : 0.f;
    if (!(x.min_p > 0.f)) x.min_p = 0.f;
    x.u = a.u[r];
    return x;
}
__device__ __forceinline__ bool usable(float t) { return t > 0.f && t < __builtin_inff(); }

__device__ __forceinline__ void no_token(const SampleArgs &a, int r)
{
    a.token[r] = -1;
    if (a.logprob) a.logprob[r] = __builtin_nanf("");
    if (a.kept_logprob) a.kept_logprob[r] = __builtin_nanf("");
}

// y: the token's logit less the largest, over t
__device__ __forceinline__ void log_probs(const SampleArgs &a, int r, double y, unsigned long long whole, unsigned long long kept)
{
    if (a.logprob) a.logprob[r] = (float)(y - log((double)whole / kUnit));
    if (a.kept_logprob) a.kept_logprob[r] = (float)(y - log((double)kept / kUnit));
}

// ---- the general way
template <bool F32>
__device__ __forceinline__ void sample_row(const SampleArgs &a, int r, RowLds &s)
{
    RowSampler<F32> x{Row<F32>(a.logits, a.stride, r, a.V), s};
    const RowAsk ask = row_ask(a, r);
    const float t = ask.t;
    // ---- the largest logit; rows without a distribution
    if (threadIdx.x == 0) {
        s.lo = 0xffffffffu;
        s.flags = 0;
    }
    RowSampler<F32>::clear(s.first);
    __syncthreads();
    {
        uint32_t top = 0xffffffffu;
        bool bad = false;
        x.row.all([&](int, float z) {
            bad |= !(z < __builtin_inff());
            top = min(top, order_key(z));
        });
        atomicMin(&s.lo, top);
        if (bad) s.flags = 1;
    }
    __syncthreads();
    x.m = key_value(s.lo);
    if (s.flags || !(x.m > -__builtin_inff()) || !usable(t)) {
        if (threadIdx.x == 0) no_token(a, r);
        return;
    }
    x.inv_t = 1.0 / (double)t;
    x.bin_scale = fminf((float)(kBins - 1) / (kWindow * t), 1e30f);
    // ---- counts and weights of the bins; the tokens that min-p leaves
    const float min_p = ask.min_p;
    uint32_t n_min = 0;
    if (threadIdx.x == 0) s.flags = 0;
    __syncthreads();
    x.row.all([&](int, float z) {
        if (z > -__builtin_inff()) {
            double w;
            const unsigned long long units = weight_of(((double)z - (double)x.m) * x.inv_t, w);
            const int b = x.bin(z);
            atomicAdd(&s.first.count[b], 1u);
            if (units) atomicAdd(&s.first.mass[b], units);
            if (min_p > 0.f && w >= (double)min_p) ++n_min;
        }
    });
    if (n_min) atomicAdd(&s.flags, n_min);
    __syncthreads();
    n_min = min_p > 0.f ? max(s.flags, 1u) : 0xffffffffu;
    // totals: the place of the last token
    x.search(s.first, 0, 0, [](uint32_t, unsigned long long) { return false; });
    uint32_t n = 0;
    unsigned long long whole = 0;
    for (int i = 0; i < kRowWaves; ++i) {
        n += s.wave_count[i];
        whole += s.wave_mass[i];
    }
    __syncthreads();
    // ---- what is kept: the first `n` tokens, of weight `kept`
    unsigned long long kept = whole;
    const auto first_tokens = [&](uint32_t k) {
        const Place p = x.find([k](uint32_t c, unsigned long long) { return c >= k; });
        n = k;
        kept = p.mass + (k - p.before) * p.each;
    };
    if (ask.k > 0 && (uint32_t)ask.k < n) first_tokens((uint32_t)ask.k);
    if (ask.top_p < 1.f && n > 1) {
        const double goal = (double)fmaxf(ask.top_p, 0.f) * (double)kept;
        const unsigned long long least = max((unsigned long long)ceil(goal), 1ull);    // (one token at least: nothing passes in front of the first)
        const Place p = x.find([least](uint32_t, unsigned long long w) { return w >= least; });
        if (p.there) {
            const double more = p.each ? ceil((goal - (double)p.mass) / (double)p.each) : 1.0;
            const uint32_t in = (uint32_t)fmin(fmax(more, 1.0), (double)p.equal);
            if (p.before + in < n) {
                n = p.before + in;
                kept = p.mass + in * p.each;
            }
        }
    }
    if (n_min < n) first_tokens(n_min);
    // ---- the token
    const double goal = (ask.u >= 0.f ? fmin((double)ask.u, 1.0) : 0.0) * (double)kept;
    const unsigned long long below = (unsigned long long)goal;
    Place p = x.find([below](uint32_t, unsigned long long w) { return w > below; });
    uint32_t nth = 0;
    if (p.there && p.before < n) {
        nth = p.each ? (uint32_t)fmin(fmax(floor((goal - (double)p.mass) / (double)p.each), 0.0), (double)(p.equal - 1)) : 0u;
        nth = min(nth, n - 1 - p.before);
    } else {        // the last one of any weight
        const unsigned long long all = kept;
        p = x.find([all](uint32_t, unsigned long long w) { return w >= all; });
        nth = (uint32_t)((kept - p.mass - 1) / p.each);
    }
    // ---- its index: the nth of those with its value.  First the run of kRowThreads pieces that holds it, then the thread, then the element.
    uint32_t *const runs = s.part.count;
    RowSampler<F32>::clear(s.part);
    __syncthreads();
    for (int i = threadIdx.x, run = 0; i < x.row.pieces; i += kRowThreads, ++run) {
        uint32_t c = 0;
        x.row.piece(i, [&](int, float z) { c += order_key(z) == p.key; });
        if (c) atomicAdd(&runs[run], c);
    }
    __syncthreads();
    x.search(s.part, 0, 0, [nth](uint32_t c, unsigned long long) { return c > nth; });
    const uint32_t run = s.found, left = nth - s.at_count;
    const int i = (int)run * kRowThreads + threadIdx.x;
    uint32_t c = 0;
    if (i < x.row.pieces) x.row.piece(i, [&](int, float z) { c += order_key(z) == p.key; });
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t ci = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(ci, o, 64);
        if (lane >= o) ci += up;
    }
    __syncthreads();
    if (lane == 63) s.wave_count[wave] = ci;
    __syncthreads();
    uint32_t before = ci - c;
    for (int j = 0; j < wave; ++j) before += s.wave_count[j];
    if (c && left >= before && left < before + c) {
        int token = -1;
        uint32_t seen = before;
        x.row.piece(i, [&](int index, float z) {
            if (order_key(z) == p.key) {
                if (seen == left) token = index;
                ++seen;
            }
        });
        a.token[r] = token;
        log_probs(a, r, ((double)key_value(p.key) - (double)x.m) * x.inv_t, whole, kept);
    }
}

// ---- 16-bit logits by value.  A pattern less kFirst, of which bits 11 to 14 are then zero, names its bin: bit 15 the sign, bits 0 to 10 the size.
constexpr uint32_t kFirst = 118 << 7;       // 2^-9
constexpr double kLowest = 128.0;           // 2^7: sixteen powers of two on
constexpr int kSide = 2048;                 // bins of a sign
constexpr int kSlots = 2 * kSide;           // of both, by size, the signs side by side
constexpr int kRare = 1024;                 // room for values of a sign below 2^-9 other than zero (one of 2800 tokens of logits that spread by 2.2)
constexpr int kRankLanes = 8, kRanked = kRowThreads / kRankLanes;   // lists up to here are sorted by counting (37 rows of 32003 29.3 -> 27.1 us)
constexpr int kFront = kRanked;             // of 32-bit logits up to here the first tokens of the order are sorted together (with top-k and top-p 36.5 -> 33.3 us)
constexpr uint32_t kNone = 0xff80ff80u;     // two -inf
constexpr int kMostParts = 32, kRuns = 8;
enum { kBad = 1, kHigh = 2, kLow = 4 };

// What the workgroup that counts a part of a row leaves of it
struct PartCounts {
    uint16_t count[2 * kSide];  // by size, the signs side by side: a part has at most 65535 tokens
    uint32_t zeros, flags, rare[2];
    unsigned long long list[2][kRare];      // key and index of the rare values, by sign: room for a whole row's, so that its way does not go by how it is cut
};

struct ChooseLds {
    uint32_t bins[2][kSlots];               // a row's quarters, two to a word (row by row); the first half: a part's counts
    unsigned long long list[3][kRare];      // the rare values by sign: key and index; 32-bit logits: those of one bin, or the order's first ones
    unsigned long long wave_mass[kRowWaves], rare_mass[2], rare_sum[kRowWaves];
    uint32_t wave_count[kRowWaves], wave_first[kRowWaves], wave_hit[2][kRowWaves];
    uint32_t rare[2], sorted[2], flags, n_min, top, zeros[kMostParts], in_bin, bin_sorted;
    uint32_t runs[kRuns];
    Place place[2][kRowWaves], spot;
    uint32_t owner;
};
union ValueLds {
    ChooseLds choose;
    RowLds row;         // for rows that take the general way
};
struct FloatLds : ChooseLds {
    alignas(16) unsigned long long mass[2 * kSide];
    double powers[64];      // 2^(j / 64)
};
static_assert(alignof(FloatLds) == 16 && sizeof(PartCounts) % 16 == 0, "cleared, written and read in 16 bytes");
union WideLds {
    FloatLds choose;
    RowLds row;
};

__device__ __forceinline__ float pattern_value(uint32_t b) { return __uint_as_float(b << 16); }
__device__ __forceinline__ uint32_t bin_pattern(int bin) { return bin < kSide ? kFirst + (uint32_t)(kSide - 1 - bin) : 0x8000u + kFirst + (uint32_t)(bin - kSide); }

// Inclusive sums over a wavefront, or over each 16 lanes of it: row shifts and two row broadcasts
#define QARL_SCAN_STEP(CTRL, ROWS) \
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false)
#define QARL_SCAN_STEP64(CTRL, ROWS) \
    v += (unsigned long long)(uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false) << 32 | \
         (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false)
template <bool WHOLE>
__device__ __forceinline__ uint32_t scan_lanes(uint32_t v)
{
    QARL_SCAN_STEP(0x111, 0xf);
    QARL_SCAN_STEP(0x112, 0xf);
    QARL_SCAN_STEP(0x114, 0xf);
    QARL_SCAN_STEP(0x118, 0xf);
    if (WHOLE) {
        QARL_SCAN_STEP(0x142, 0xa);
        QARL_SCAN_STEP(0x143, 0xc);
    }
    return v;
}
template <bool WHOLE>
__device__ __forceinline__ unsigned long long scan_lanes(unsigned long long v)
{
    QARL_SCAN_STEP64(0x111, 0xf);
    QARL_SCAN_STEP64(0x112, 0xf);
    QARL_SCAN_STEP64(0x114, 0xf);
    QARL_SCAN_STEP64(0x118, 0xf);
    if (WHOLE) {
        QARL_SCAN_STEP64(0x142, 0xa);
        QARL_SCAN_STEP64(0x143, 0xc);
    }
    return v;
}
#undef QARL_SCAN_STEP
#undef QARL_SCAN_STEP64
__device__ __forceinline__ uint32_t lane_of(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ unsigned long long lane_of(unsigned long long v, int lane)
{
    return (unsigned long long)lane_of((uint32_t)(v >> 32), lane) << 32 | lane_of((uint32_t)v, lane);
}

// Eight values into the bins (`bump` to be added to their counts), or to what is kept of others
struct Counts {
    uint32_t *bins, *rare;
    unsigned long long *list;
    uint32_t room, zeros, flags;
    __device__ __forceinline__ void pair(uint32_t w, int index, uint32_t bump)
    {
        typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
        const u16x2 r = __builtin_bit_cast(u16x2, w) - (u16x2){(uint16_t)kFirst, (uint16_t)kFirst};
        const uint32_t slot = __builtin_bit_cast(uint32_t, (u16x2)(r << 1)) | __builtin_bit_cast(uint32_t, (u16x2)(r >> 15));
        const uint32_t rw = __builtin_bit_cast(uint32_t, r);
        if ((rw & 0x78007800u) == 0) {
            atomicAdd(bins + (slot & 0xffffu), bump);
            atomicAdd(bins + (slot >> 16), bump);
            return;
        }
        if (w == kNone) return;
#pragma unroll 1
        for (int e = 0; e < 2; ++e) {
            const uint32_t b = (w >> 16 * e) & 0xffffu, size = b & 0x7fffu;
            if (((b - kFirst) & 0x7800u) == 0) {
                atomicAdd(bins + ((slot >> 16 * e) & 0xffffu), bump);
            } else if (size == 0) {
                ++zeros;
            } else if (size < kFirst) {
                const uint32_t at = atomicAdd(rare + (b >> 15), 1u);
                if (at < room) list[(b >> 15) * room + at] = (unsigned long long)order_key(pattern_value(b)) << 32 | (uint32_t)(index + e);
            } else if (b != 0xff80u) {
                flags |= size >= 0x7f80u ? kBad : b & 0x8000u ? kLow : kHigh;
            }
        }
    }
    __device__ __forceinline__ void piece(u32x4 w, int first, int V, uint32_t bump)
    {
        if (first < 0 || first + 8 > V) {       // those outside the row become -inf
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if ((unsigned)(first + e) >= (unsigned)V) w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | (kNone & 0xffff0000u) : (w[e >> 1] & 0xffff0000u) | (kNone & 0xffffu);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) pair(w[e], first + 2 * e, bump);
    }
};

struct Chosen {
    uint32_t key;           // the token's value
    uint32_t nth;           // of the tokens with that value; of one out of a list: its index
    bool listed, none;
};

// What the counts of a row say.  Thread i holds bins 4 i .. 4 i + 3 of the order: positive values falling, then negative ones; the rare ones and zero stand between.
template <bool F32>
struct Chooser {
    using Lds = typename std::conditional<F32, FloatLds, ChooseLds>::type;
    static constexpr int kEach = 2 * kSide / kRowThreads;
    Lds &s;
    const Row<F32> &row;
    uint32_t c[kEach], upto[kEach];                 // tokens of the bins, and of the order up to their ends
    unsigned long long unit[kEach], mass[kEach];    // a token's weight (32-bit logits: the bin's), and that of the order up to the bins' ends
    uint32_t positive, special[3];              // tokens of the positive bins; of the rare positive values, of zero, of the rare negative ones
    unsigned long long positive_mass, special_mass[3], zero_unit;
    float m;
    double inv_t;
    int calls;
    uint32_t list_before, list_count;           // 32-bit logits: the tokens of the order that are in the third list
    unsigned long long list_mass;
    bool lost;                                  // 32-bit logits: sixteen keys' tokens are more than there is room for

    // 32-bit logits are weighed one by one: y = k ln 2 / 64 + r, the power series of e^r up to r^4 within 4e-14, 2^(k / 64) out of a table.  (y below -31: no unit.)
    __device__ static __forceinline__ unsigned long long weigh_by(const Lds &s, double y, double &w)
    {
        if constexpr (!F32) return weight_of(y, w);
        else {
            if (!(y > -31.5)) {
                w = 0.0;
                return 0;
            }
            const double kd = rint(y * 92.332482616893656877);
            const double r = fma(-kd, 0.010830424696249145, y);
            const int k = (int)kd;
            double p = fma(1.0 / 24.0, r, 1.0 / 6.0);
            p = fma(p, r, 0.5);
            p = fma(p, r, 1.0);
            p = fma(p, r, 1.0);
            p *= s.powers[k & 63];
            w = __longlong_as_double(__double_as_longlong(p) + ((long long)(k >> 6) << 52));
            return weight_units(w);
        }
    }
    __device__ __forceinline__ unsigned long long weigh(float z, double &w) const { return weigh_by(s, ((double)z - (double)m) * inv_t, w); }

    // The place among the n <= kRowThreads tokens of a list of keys and indices, each a bin of its own: sorted the first time that one is asked for.
    // (The result in s.spot, its index in s.owner.  A function of its own: it is seldom called, and costs the others registers.)
    template <typename Fn>
    __device__ static __attribute__((noinline)) void among(Lds &s, unsigned long long *list, uint32_t n, uint32_t *sorted, uint32_t before, unsigned long long mass, float m,
                                                           double inv_t, Fn pass)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        __syncthreads();
        if (!*sorted && n <= (uint32_t)kRanked) {       // eight lanes count what stands in front of a token
            const uint32_t token = threadIdx.x / kRankLanes;
            const unsigned long long x = token < n ? list[token] : 0;
            uint32_t rank = 0;
            if ((uint32_t)(wave * 64 / kRankLanes) < n) {
                for (uint32_t j = threadIdx.x % kRankLanes; j < n; j += kRankLanes) rank += list[j] < x;
#pragma unroll
                for (int o = kRankLanes / 2; o > 0; o >>= 1) rank += (uint32_t)__shfl_xor((int)rank, o, 64);
            }
            __syncthreads();
            if (token < n && threadIdx.x % kRankLanes == 0) list[rank] = x;
            __syncthreads();
            if (threadIdx.x == 0) *sorted = 1;
        } else if (!*sorted) {
            uint32_t size = 2;
            while (size < n) size *= 2;
            if (threadIdx.x >= n && threadIdx.x < size) list[threadIdx.x] = ~0ull;
            for (uint32_t k = 2; k <= size; k *= 2) {
                for (uint32_t j = k / 2; j > 0; j /= 2) {
                    __syncthreads();
                    if (threadIdx.x < size / 2) {
                        const uint32_t t = threadIdx.x, a = 2 * t - (t & (j - 1)), b = a + j;
                        const unsigned long long x = list[a], y = list[b];
                        if ((x > y) == ((a & k) == 0)) {
                            list[a] = y;
                            list[b] = x;
                        }
                    }
                }
            }
            __syncthreads();
            if (threadIdx.x == 0) *sorted = 1;
        }
        uint32_t key = 0, index = 0;
        unsigned long long u = 0;
        if (threadIdx.x < n) {
            index = (uint32_t)list[threadIdx.x];
            key = (uint32_t)(list[threadIdx.x] >> 32);
            double w;
            u = weigh_by(s, ((double)key_value(key) - (double)m) * inv_t, w);
        }
        const unsigned long long upto = scan_lanes<true>(u);
        if (lane == 63) s.rare_sum[wave] = upto;
        __syncthreads();
        const unsigned long long sums = s.rare_sum[lane & (kRowWaves - 1)], sums_upto = scan_lanes<false>(sums);
        const int at = __builtin_amdgcn_readfirstlane(wave);
        mass += upto - u + lane_of(sums_upto, at) - lane_of(sums, at);
        before += threadIdx.x;
        // the first that passes: what stands in front of it does not
        if (threadIdx.x < n && pass(before + 1, mass + u) && (threadIdx.x == 0 || !pass(before, mass))) {
            s.spot = Place{key, before, 1, mass, u, true};
            s.owner = index;
        }
        __syncthreads();
    }

    // 32-bit logits, a bin of more tokens than there is room for: counted again by the next twelve bits of their keys.  The sixteen keys in which the place
    // lies in s.spot, the first of them as its key, their weight in place of one's.
    template <typename Fn>
    __device__ static __attribute__((noinline)) void narrow(Lds &s, Row<F32> row, uint32_t lo, uint32_t before, unsigned long long mass, float m, double inv_t, Fn pass)
    {
        if constexpr (F32) {
            const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = (int)threadIdx.x * kEach;
            static_assert(kEach == 4 && 16 * kEach * kRowThreads == 1 << 16, "a bin's keys");
            *(u32x4 *)(s.bins[0] + first) = ((u32x4 *)(s.mass + first))[0] = ((u32x4 *)(s.mass + first))[1] = u32x4{0, 0, 0, 0};
            __syncthreads();
            row.all([&](int, float z) {
                const uint32_t k = order_key(z) - lo;
                if (k >> 16 == 0) {
                    double w;
                    const unsigned long long units = weigh_by(s, ((double)z - (double)m) * inv_t, w);
                    atomicAdd(&s.bins[0][k >> 4], 1u);
                    if (units) atomicAdd(&s.mass[k >> 4], units);
                }
            });
            __syncthreads();
            uint32_t csum = 0;
            unsigned long long wsum = 0;
            for (int i = 0; i < kEach; ++i) {
                csum += s.bins[0][first + i];
                wsum += s.mass[first + i];
            }
            const uint32_t ci = scan_lanes<true>(csum);
            const unsigned long long wi = scan_lanes<true>(wsum);
            if (lane == 63) {
                s.wave_count[wave] = ci;
                s.wave_mass[wave] = wi;
            }
            __syncthreads();
            const uint32_t wc = s.wave_count[lane & (kRowWaves - 1)], wcs = scan_lanes<false>(wc);
            const unsigned long long wm = s.wave_mass[lane & (kRowWaves - 1)], wms = scan_lanes<false>(wm);
            const int at = __builtin_amdgcn_readfirstlane(wave);
            before += ci - csum + lane_of(wcs, at) - lane_of(wc, at);
            mass += wi - wsum + lane_of(wms, at) - lane_of(wm, at);
            for (int i = 0; i < kEach; ++i) {
                const uint32_t n = s.bins[0][first + i];
                const unsigned long long w = s.mass[first + i];
                if (n && pass(before + n, mass + w) && !pass(before, mass)) s.spot = Place{lo + 16 * (uint32_t)(first + i), before, n, mass, w, true};
                before += n;
                mass += w;
            }
            __syncthreads();
        }
    }

    // 32-bit logits: the tokens of keys lo .. hi (a bin, or sixteen of its keys) into the third list; a few of them with all that stand in front, for later places
    // lie further in front.  (The last that was done with the list ended with a barrier.)
    __device__ __forceinline__ void gather(const Place &bin, uint32_t lo, uint32_t hi, bool last)
    {
        if (bin.before >= list_before && bin.before + bin.equal <= list_before + list_count) return;        // (they are there)
        const bool all = !last && bin.before + bin.equal <= (uint32_t)kFront;
        list_before = all ? 0 : bin.before;
        list_count = all ? bin.before + bin.equal : bin.equal;
        list_mass = all ? 0 : bin.mass;
        if (all) lo = 0;
        if (threadIdx.x == 0) s.in_bin = s.bin_sorted = 0;
        __syncthreads();
        row.all([&](int index, float z) {
            const uint32_t k = order_key(z);
            if (k >= lo && k <= hi) {
                const uint32_t at = atomicAdd(&s.in_bin, 1u);
                if (at < (uint32_t)kRare) s.list[2][at] = (unsigned long long)k << 32 | (uint32_t)index;
            }
        });
        __syncthreads();
    }

    template <typename Fn>
    __device__ __forceinline__ Place find(Fn pass, bool &listed, bool last = false)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = calls++ & 1;     // (what the call before has found may still be read)
        bool hit_here = false;
        Place mine;
#pragma unroll
        for (int i = kEach - 1; i >= 0; --i)
            if (c[i] && pass(upto[i], mass[i])) {
                hit_here = true;
                mine = Place{bin_pattern(threadIdx.x * kEach + i), upto[i], c[i], mass[i], unit[i], true};
            }
        const unsigned long long hit = __ballot(hit_here);
        if (lane == 0) s.wave_hit[half][wave] = hit != 0;
        if (hit && lane == __ffsll((long long)hit) - 1) {
            mine.before -= mine.equal;
            mine.mass -= F32 ? mine.each : mine.equal * mine.each;
            s.place[half][wave] = mine;
        }
        __syncthreads();
        const uint32_t hits = (uint32_t)__ballot(lane < kRowWaves && s.wave_hit[half][lane & (kRowWaves - 1)] != 0);
        listed = false;
        if (!(hits & 0xffu)) {
            uint32_t b = positive;          // between the signs
            unsigned long long w = positive_mass;
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                if (special[j] && pass(b + special[j], w + special_mass[j])) {
                    if (j == 1) return Place{order_key(0.f), b, special[1], w, zero_unit, true};
                    listed = true;
                    among(s, s.list[j >> 1], special[j], &s.sorted[j >> 1], b, w, m, inv_t, pass);
                    return s.spot;
                }
                b += special[j];
                w += special_mass[j];
            }
            if (!hits) return Place{};
        }
        Place p = s.place[half][__ffs((int)hits) - 1];
        if (F32) {
            const uint32_t one = p.key << 16 ^ (p.key >> 15 ? 0u : 0x7fffffffu), other = one ^ 0xffffu;
            uint32_t lo = min(one, other), hi = max(one, other);
            if (p.equal > (uint32_t)kRare) {
                narrow(s, row, lo, p.before, p.mass, m, inv_t, pass);
                p = s.spot;
                lo = p.key;
                hi = lo + 15;
                if (p.equal > (uint32_t)kRare) {
                    lost = true;
                    return p;
                }
            }
            gather(p, lo, hi, last);
            listed = true;
            among(s, s.list[2], list_count, &s.bin_sorted, list_before, list_mass, m, inv_t, pass);
            return s.spot;
        }
        p.key = order_key(pattern_value(p.key));
        return p;
    }

    // False where the row has to take the general way.  Writes the log-probs.  32-bit logits: the largest one's key is s.top, the bins' weights are s.mass.
    __device__ __forceinline__ bool choose(const SampleArgs &a, int r, const RowAsk &ask, uint32_t zeros, Chosen &out)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & (kRowWaves - 1);
        calls = 0;
        lost = false;
        list_before = list_count = 0;
        const uint32_t n_rare[2] = {min(s.rare[0], (uint32_t)kRare), min(s.rare[1], (uint32_t)kRare)};
        double w = 0.0;
        uint32_t csum = 0;
        unsigned long long wsum = 0;
        out.none = true;
        if (!F32) {
            // ---- the largest value
            int first = kEach;
#pragma unroll
            for (int i = kEach - 1; i >= 0; --i)
                if (c[i]) first = i;
            const unsigned long long some = __ballot(first < kEach);
            if (lane == (some ? __ffsll((long long)some) - 1 : 0)) s.wave_first[wave] = some ? threadIdx.x * kEach + first : 0xffffffffu;
            __syncthreads();
            if ((s.flags & kBad) || !usable(ask.t)) return true;
            if ((s.flags & kHigh) || s.rare[0] > (uint32_t)kRare || s.rare[1] > (uint32_t)kRare) return false;
            const uint32_t tops = s.wave_first[l16], with = (uint32_t)__ballot(lane < kRowWaves && tops != 0xffffffffu);
            if (with & 0xffu) m = pattern_value(bin_pattern((int)lane_of(tops, __ffs((int)with) - 1)));
            else if (n_rare[0] || (!zeros && n_rare[1])) {      // a rare one
                const int sign = !n_rare[0];
                if (threadIdx.x < n_rare[sign]) atomicMin(&s.top, (uint32_t)(s.list[sign][threadIdx.x] >> 32));
                __syncthreads();
                m = key_value(s.top);
            } else if (zeros) m = 0.f;
            else if (with) m = pattern_value(bin_pattern((int)lane_of(tops, __ffs((int)with) - 1)));
            else return !(s.flags & kLow);      // (only -inf: no token)
            inv_t = 1.0 / (double)ask.t;
            if ((s.flags & kLow) && ((double)m + kLowest) * inv_t < 31.0) return false;     // those of -128 and less weigh a unit or more
            // ---- weights.  A thread's values lie a step apart: the first one's weight by the exponential, the others by a factor
            uint32_t above = 0;
            double factor = 0.0;
            if (first < kEach) {
                const uint32_t b = bin_pattern(threadIdx.x * kEach + first);
                const float z = pattern_value(b), next = pattern_value(b + (b >> 15 ? 1 : -1));
                weigh(z, w);
                weight_of(((double)next - (double)z) * inv_t, factor);
            }
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (i > first) w *= factor;
                unit[i] = c[i] ? weight_units(w) : 0;
                above += w >= (double)ask.min_p ? c[i] : 0;
                csum += c[i];
                wsum += c[i] * unit[i];
            }
#pragma unroll
            for (int sign = 0; sign < 2; ++sign) {
                if ((uint32_t)(wave * 64) < n_rare[sign]) {
                    unsigned long long units = 0;
                    if (threadIdx.x < n_rare[sign]) {
                        units = weigh(key_value((uint32_t)(s.list[sign][threadIdx.x] >> 32)), w);
                        above += w >= (double)ask.min_p;
                    }
                    units = scan_lanes<true>(units);
                    if (lane == 63) atomicAdd(&s.rare_mass[sign], units);
                }
            }
            zero_unit = 0;
            if (zeros) {
                zero_unit = weigh(0.f, w);
                if (threadIdx.x == 0 && w >= (double)ask.min_p) above += zeros;
            }
            if (ask.min_p > 0.f && above) atomicAdd(&s.n_min, above);
        } else {
            if ((s.flags & kHigh) || s.rare[0] > (uint32_t)kRare || s.rare[1] > (uint32_t)kRare) return false;
            if ((s.flags & kLow) && ((double)m + kLowest) * inv_t < 31.0) return false;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                csum += c[i];
                wsum += unit[i];
            }
            zero_unit = zeros ? weigh(0.f, w) : 0;
        }
        special[0] = n_rare[0];
        special[1] = zeros;
        special[2] = n_rare[1];
        const uint32_t ci = scan_lanes<true>(csum);
        const unsigned long long wi = scan_lanes<true>(wsum);
        if (lane == 63) {
            s.wave_count[wave] = ci;
            s.wave_mass[wave] = wi;
        }
        __syncthreads();
        special_mass[0] = s.rare_mass[0];
        special_mass[1] = special[1] * zero_unit;
        special_mass[2] = s.rare_mass[1];
        const uint32_t wc = s.wave_count[l16], wcs = scan_lanes<false>(wc);
        const unsigned long long wm = s.wave_mass[l16], wms = scan_lanes<false>(wm);
        positive = lane_of(wcs, kRowWaves / 2 - 1);
        positive_mass = lane_of(wms, kRowWaves / 2 - 1);
        uint32_t n = special[0] + special[1] + special[2];
        unsigned long long whole = special_mass[0] + special_mass[1] + special_mass[2];
        const int at = __builtin_amdgcn_readfirstlane(wave);
        uint32_t cb = ci - csum + lane_of(wcs, at) - lane_of(wc, at) + (at >= kRowWaves / 2 ? n : 0);
        unsigned long long mb = wi - wsum + lane_of(wms, at) - lane_of(wm, at) + (at >= kRowWaves / 2 ? whole : 0);
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            upto[i] = cb += c[i];
            mass[i] = mb += F32 ? unit[i] : c[i] * unit[i];
        }
        n += lane_of(wcs, kRowWaves - 1);
        whole += lane_of(wms, kRowWaves - 1);
        // ---- what is kept, and the token
        unsigned long long kept = whole;
        bool listed;
        const auto first_tokens = [&](uint32_t k) {
            const Place p = find([k](uint32_t x, unsigned long long) { return x >= k; }, listed);
            n = k;
            kept = p.mass + (k - p.before) * p.each;
        };
        if (ask.k > 0 && (uint32_t)ask.k < n) first_tokens((uint32_t)ask.k);
        if (F32 && lost) return false;
        if (ask.top_p < 1.f && n > 1) {
            const double goal = (double)fmaxf(ask.top_p, 0.f) * (double)kept;
            const unsigned long long least = max((unsigned long long)ceil(goal), 1ull);    // (one token at least: nothing passes in front of the first)
            const Place p = find([least](uint32_t, unsigned long long x) { return x >= least; }, listed);
            if (F32 && lost) return false;
            if (p.there) {
                const double more = p.each ? ceil((goal - (double)p.mass) / (double)p.each) : 1.0;
                const uint32_t in = (uint32_t)fmin(fmax(more, 1.0), (double)p.equal);
                if (p.before + in < n) {
                    n = p.before + in;
                    kept = p.mass + in * p.each;
                }
            }
        }
        const uint32_t n_min = ask.min_p > 0.f ? max(s.n_min, 1u) : 0xffffffffu;
        if (n_min < n) first_tokens(n_min);
        if (F32 && lost) return false;
        const double goal = (ask.u >= 0.f ? fmin((double)ask.u, 1.0) : 0.0) * (double)kept;
        const unsigned long long below = (unsigned long long)goal;
        Place p = find([below](uint32_t, unsigned long long x) { return x > below; }, listed, true);
        if (F32 && lost) return false;
        if (p.there && p.before < n) {
            out.nth = p.each ? (uint32_t)fmin(fmax(floor((goal - (double)p.mass) / (double)p.each), 0.0), (double)(p.equal - 1)) : 0u;
            out.nth = min(out.nth, n - 1 - p.before);
        } else {        // the last one of any weight
            const unsigned long long all = kept;
            p = find([all](uint32_t, unsigned long long x) { return x >= all; }, listed, true);
            if (F32 && lost) return false;
            out.nth = (uint32_t)((kept - p.mass - 1) / p.each);
        }
        if (listed) out.nth = s.owner;
        out.key = p.key;
        out.listed = listed;
        out.none = false;
        if (threadIdx.x == kRowThreads - 1) log_probs(a, r, ((double)key_value(p.key) - (double)m) * inv_t, whole, kept);     // (while the token is looked for)
        return true;
    }
};

__device__ __forceinline__ void clear_choice(ChooseLds &s)
{
    if (threadIdx.x < kMostParts) s.zeros[threadIdx.x] = 0;
    if (threadIdx.x < kRuns) s.runs[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        s.rare[0] = s.rare[1] = s.flags = s.n_min = s.sorted[0] = s.sorted[1] = 0;
        s.rare_mass[0] = s.rare_mass[1] = 0;
        s.top = 0xffffffffu;
    }
}

// The index of the nth token with that pattern among pieces [from, to), at most NR runs of kRowThreads.  First the run, then the thread, then the element.
template <int NR>
__device__ __forceinline__ void answer(const SampleArgs &a, int r, const Row<false> &row, int from, int to, uint32_t nth, uint32_t pattern, ChooseLds &s)
{
    static_assert(NR <= kRuns, "room for the runs");
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint32_t keep = pattern ? 0xffffffffu : 0x7fff7fffu, both = pattern | pattern << 16;      // (zeros of either sign)
    u32x4 w[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        w[i] = u32x4{~both, ~both, ~both, ~both};
        if (from + i * kRowThreads + tid < to) w[i] = row.base[from + i * kRowThreads + tid];
    }
    // the top bit of each half that matches
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    const auto same = [&](uint32_t v) {
        const uint32_t x = (v ^ both) & keep;
        return __builtin_bit_cast(uint32_t, (u16x2)(__builtin_bit_cast(u16x2, x) - (u16x2){1, 1})) & ~x & 0x80008000u;
    };
    const auto inside = [&](int i) {        // of the piece's eight elements those in the row
        const int first = (from + i * kRowThreads + tid) * 8 - row.off;
        return (first < 0 ? 0xffu << min(-first, 8) : 0xffu) & (first + 8 > row.V ? 0xffu >> min(first + 8 - row.V, 8) : 0xffu);
    };
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        uint32_t n = __popc(same(w[i][0])) + __popc(same(w[i][1])) + __popc(same(w[i][2])) + __popc(same(w[i][3]));
        if (n) {
            const uint32_t in = inside(i);
            if (in != 0xffu) {
                n = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e) n += (same(w[i][e >> 1]) >> (e & 1 ? 31 : 15) & in >> e) & 1u;
            }
            if (n) atomicAdd(&s.runs[i], n);
        }
    }
    __syncthreads();
    int run = 0;
    u32x4 its = w[0];
    uint32_t count = s.runs[0];
#pragma unroll
    for (int i = 1; i < NR; ++i) {
        const uint32_t here = s.runs[i];
        if (run == i - 1 && nth >= count) {
            nth -= count;
            count = here;
            run = i;
            its = w[i];
        }
    }
    uint32_t mine = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t m = same(its[e]);
        mine |= (m >> 15 & 1u) << (2 * e) | (m >> 31) << (2 * e + 1);
    }
    mine &= inside(run);
    const uint32_t in = (uint32_t)__popc(mine), upto = scan_lanes<true>(in);
    if (lane == 63) s.wave_first[wave] = upto;
    __syncthreads();
    const uint32_t wc = s.wave_first[lane & (kRowWaves - 1)], wcs = scan_lanes<false>(wc);
    const int at = __builtin_amdgcn_readfirstlane(wave);
    const uint32_t before = upto - in + lane_of(wcs, at) - lane_of(wc, at);
    if (nth >= before && nth < before + in) {
        for (uint32_t j = before; j < nth; ++j) mine &= mine - 1;
        a.token[r] = (from + run * kRowThreads + tid) * 8 - row.off + __ffs((int)mine) - 1;
    }
}

// A workgroup takes a row: each quarter NQ pieces of 16 bytes a thread, the next one's requested while one is counted.
template <int NQ>
__global__ __launch_bounds__(kRowThreads) void sample_values_kernel(SampleArgs a)
{
    extern __shared__ __align__(16) char lds[];
    ChooseLds &s = ((ValueLds *)lds)->choose;
    const int r = blockIdx.x, tid = (int)threadIdx.x;
    const Row<false> row(a.logits, a.stride, r, a.V);
    const int quarter = (row.pieces + 3) / 4;
    u32x4 w[2][NQ];
    const auto load = [&](int q, int to) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int in = i * kRowThreads + tid;
            w[to][i] = u32x4{kNone, kNone, kNone, kNone};
            if (in < quarter && q * quarter + in < row.pieces) w[to][i] = row.base[q * quarter + in];
        }
    };
    load(0, 0);
    const RowAsk ask = row_ask(a, r);
    for (int i = tid; i < 2 * kSlots / 4; i += kRowThreads) ((u32x4 *)s.bins)[i] = u32x4{0, 0, 0, 0};
    clear_choice(s);
    __syncthreads();
    Counts counts{nullptr, s.rare, s.list[0], kRare, 0, 0};
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {      // (a loop: the way of every piece is long, and the instruction cache small)
        counts.bins = s.bins[half];
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            const int q = 2 * half + odd;
            if (q < 3) load(q + 1, odd ^ 1);
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                const int in = i * kRowThreads + tid;
                if (in < quarter) counts.piece(w[odd][i], (q * quarter + in) * 8 - row.off, a.V, odd ? 65536u : 1u);
            }
            if (counts.zeros) atomicAdd(&s.zeros[q], counts.zeros);
            counts.zeros = 0;
        }
    }
    if (counts.flags) atomicOr(&s.flags, counts.flags);
    __syncthreads();
    Chooser<false> x{s, row};
    {
        const bool negative = tid >= kRowThreads / 2;
        const int size = negative ? (tid - kRowThreads / 2) * 4 : kSide - 4 - tid * 4;      // of the smallest of the thread's four
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int at = 2 * (size + (negative ? i : 3 - i)) + negative;
            const uint32_t lo = s.bins[0][at], hi = s.bins[1][at];
            x.c[i] = (lo & 0xffffu) + (lo >> 16) + (hi & 0xffffu) + (hi >> 16);
        }
    }
    const uint32_t zeros[4] = {s.zeros[0], s.zeros[1], s.zeros[2], s.zeros[3]};
    Chosen got;
    if (!x.choose(a, r, ask, zeros[0] + zeros[1] + zeros[2] + zeros[3], got)) {
        __syncthreads();
        sample_row<false>(a, r, ((ValueLds *)lds)->row);
        return;
    }
    if (got.none || got.listed) {
        if (tid == 0) {
            if (got.none) no_token(a, r);
            else a.token[r] = (int)got.nth;
        }
        return;
    }
    const uint32_t pattern = __float_as_uint(key_value(got.key)) >> 16;
    const uint32_t at = pattern ? 2 * ((pattern & 0x7fffu) - kFirst) + (pattern >> 15) : 0, lo = s.bins[0][at], hi = s.bins[1][at];
    const uint32_t n[3] = {pattern ? lo & 0xffffu : zeros[0], pattern ? lo >> 16 : zeros[1], pattern ? hi & 0xffffu : zeros[2]};
    uint32_t nth = got.nth;
    int q = 0;
    while (q < 3 && nth >= n[q]) nth -= n[q++];
    answer<NQ>(a, r, row, q * quarter, min((q + 1) * quarter, row.pieces), nth, pattern, s);
}

// Few rows: each cut into parts, counted by workgroups of their own ...
constexpr int kCountThreads = 512;
__global__ __launch_bounds__(kCountThreads) void sample_count_kernel(SampleArgs a, int parts)
{
    __shared__ __align__(16) uint32_t bins[kSlots];
    __shared__ unsigned long long list[2][kRare];
    __shared__ uint32_t rare[2], zeros, flags;
    const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = (int)threadIdx.x;
    const Row<false> row(a.logits, a.stride, r, a.V);
    const int per = (row.pieces + parts - 1) / parts, from = part * per, to = min(from + per, row.pieces);
    constexpr int kAhead = 4;
    u32x4 w[kAhead];
    const auto load = [&](int i0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            w[i] = u32x4{kNone, kNone, kNone, kNone};
            if (i0 + i * kCountThreads + tid < to) w[i] = row.base[i0 + i * kCountThreads + tid];
        }
    };
    load(from);
    for (int i = tid; i < kSide / 2; i += kCountThreads) ((u32x4 *)bins)[i] = u32x4{0, 0, 0, 0};
    if (tid == 0) rare[0] = rare[1] = zeros = flags = 0;
    __syncthreads();
    Counts counts{bins, rare, list[0], kRare, 0, 0};
    for (int i0 = from; i0 < to; i0 += kAhead * kCountThreads) {
        if (i0 > from) load(i0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) counts.piece(w[i], (i0 + i * kCountThreads + tid) * 8 - row.off, a.V, 1u);
    }
    if (counts.zeros) atomicAdd(&zeros, counts.zeros);
    if (counts.flags) atomicOr(&flags, counts.flags);
    __syncthreads();
    PartCounts &out = ((PartCounts *)a.ws)[blockIdx.x];
    for (int i = tid; i < kSide / 4; i += kCountThreads) {      // eight counts of 16 bits
        const u32x4 x = ((const u32x4 *)bins)[2 * i], y = ((const u32x4 *)bins)[2 * i + 1];
        ((u32x4 *)out.count)[i] = u32x4{x[0] | x[1] << 16, x[2] | x[3] << 16, y[0] | y[1] << 16, y[2] | y[3] << 16};
    }
    if (tid == 0) *(u32x4 *)&out.zeros = u32x4{zeros, flags, rare[0], rare[1]};
    for (int sign = 0; sign < 2; ++sign)
        for (uint32_t i = tid; i < min(rare[sign], (uint32_t)kRare); i += kCountThreads) out.list[sign][i] = list[sign][i];
}

// ... and put together by one, which chooses and looks for the token in the part that holds it
template <int NR>
__global__ __launch_bounds__(kRowThreads) void sample_choose_kernel(SampleArgs a, int parts)
{
    extern __shared__ __align__(16) char lds[];
    ChooseLds &s = ((ValueLds *)lds)->choose;
    const int r = blockIdx.x, tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Row<false> row(a.logits, a.stride, r, a.V);
    const PartCounts *const of = (const PartCounts *)a.ws + (int64_t)r * parts;
    const RowAsk ask = row_ask(a, r);
    // everything is requested at once: a wavefront's parts' heads, the beginnings of their lists (what may not be there is not used), and thread i's four bins,
    // the even or the odd ones of eight counts
    constexpr int kWaveParts = kMostParts / kRowWaves;
    u32x4 head[kWaveParts];     // zeros, flags, rare values of either sign
    unsigned long long early[kWaveParts][2];
#pragma unroll
    for (int i = 0; i < kWaveParts; ++i) {
        const int p = wave + i * kRowWaves;
        head[i] = u32x4{0, 0, 0, 0};
        early[i][0] = early[i][1] = 0;
        if (p < parts) {
            head[i] = *(const u32x4 *)&of[p].zeros;
            early[i][0] = of[p].list[0][lane];
            early[i][1] = of[p].list[1][lane];
        }
    }
    const bool negative = tid >= kRowThreads / 2;
    const int eight = negative ? tid - kRowThreads / 2 : kRowThreads / 2 - 1 - tid;
    uint32_t c[4] = {0, 0, 0, 0};
#pragma unroll 1
    for (int p0 = 0; p0 < parts; p0 += 8) {
        u32x4 w[8];
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            w[p] = u32x4{0, 0, 0, 0};
            if (p0 + p < parts) w[p] = ((const u32x4 *)of[p0 + p].count)[eight];
        }
        if (p0 == 0) clear_choice(s);
#pragma unroll
        for (int p = 0; p < 8; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] += negative ? w[p][i] >> 16 : w[p][i] & 0xffffu;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kWaveParts; ++j) {
        const int p = wave + j * kRowWaves;
        if (p >= parts) break;
        if (lane == 0) {
            s.zeros[p] = head[j][0];
            if (head[j][1]) atomicOr(&s.flags, head[j][1]);
        }
#pragma unroll
        for (int sign = 0; sign < 2; ++sign) {
            const uint32_t n = head[j][2 + sign];
            if (n == 0) continue;
            uint32_t base = 0;
            if (lane == 0) base = atomicAdd(&s.rare[sign], n <= (uint32_t)kRare ? n : (uint32_t)kRare + 1);
            base = lane_of(base, 0);
            if (n > (uint32_t)kRare) continue;
            for (uint32_t i = lane; i < n; i += 64)
                if (base + i < (uint32_t)kRare) s.list[sign][base + i] = i < 64 ? early[j][sign] : of[p].list[sign][i];
        }
    }
    __syncthreads();
    Chooser<false> x{s, row};
#pragma unroll
    for (int i = 0; i < 4; ++i) x.c[i] = negative ? c[i] : c[3 - i];
    const uint32_t zeros_here = lane < parts && lane < kMostParts ? s.zeros[lane & (kMostParts - 1)] : 0, zeros_upto = scan_lanes<true>(zeros_here);
    Chosen got;
    if (!x.choose(a, r, ask, lane_of(zeros_upto, 63), got)) {
        __syncthreads();
        sample_row<false>(a, r, ((ValueLds *)lds)->row);
        return;
    }
    if (got.none || got.listed) {
        if (tid == 0) {
            if (got.none) no_token(a, r);
            else a.token[r] = (int)got.nth;
        }
        return;
    }
    // the part: lane p has its tokens of that value
    const uint32_t pattern = __float_as_uint(key_value(got.key)) >> 16;
    uint32_t in = zeros_here;
    if (pattern) in = lane < parts ? of[lane].count[2 * ((pattern & 0x7fffu) - kFirst) + (pattern >> 15)] : 0;
    const uint32_t upto = scan_lanes<true>(in);
    const int part = __ffsll((long long)__ballot(upto > got.nth)) - 1;
    const int per = (row.pieces + parts - 1) / parts;
    answer<NR>(a, r, row, part * per, min((part + 1) * per, row.pieces), got.nth - (lane_of(upto, part) - lane_of(in, part)), pattern, s);
}

// ---- 32-bit logits: a row is read for its largest logit, for the bins, and for the tokens of each bin that a place is sought in.

// Pieces [from, to): the key of the largest logit into s.top, and whether there is a NaN or +inf into s.flags
__device__ __forceinline__ void float_top(const Row<true> &row, int from, int to, FloatLds &s)
{
    uint32_t top = 0xffffffffu;
    bool bad = false;
    row.span(from, to, [&](int, float z) {
        bad |= !(z < __builtin_inff());
        top = min(top, order_key(z));
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = min(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if ((threadIdx.x & 63) == 0) atomicMin(&s.top, top);
    if (bad) s.flags = kBad;
}

// Pieces [from, to) into the bins
__device__ __forceinline__ void float_bins(const Row<true> &row, int from, int to, float min_p, const Chooser<true> &x, FloatLds &s)
{
    uint32_t zeros = 0, flags = 0, above = 0;
    row.span(from, to, [&](int index, float z) {
        const uint32_t bits = __float_as_uint(z), b = bits >> 16, rb = (b - kFirst) & 0xffffu;
        if (z == -__builtin_inff()) return;
        double w;
        const unsigned long long units = x.weigh(z, w);
        above += w >= (double)min_p;
        if ((rb & 0x7800u) == 0) {
            const uint32_t slot = 2 * (rb & 0x7fffu) + (rb >> 15);
            atomicAdd(&s.bins[0][slot], 1u);
            if (units) atomicAdd(&s.mass[slot], units);
        } else if ((bits & 0x7fffffffu) == 0) {
            ++zeros;
        } else if ((b & 0x7fffu) < kFirst) {
            const uint32_t at = atomicAdd(&s.rare[b >> 15], 1u);
            if (at < (uint32_t)kRare) s.list[b >> 15][at] = (unsigned long long)order_key(z) << 32 | (uint32_t)index;
            atomicAdd(&s.rare_mass[b >> 15], units);
        } else {
            flags |= b & 0x8000u ? kLow : kHigh;
        }
    });
    if (zeros) atomicAdd(&s.zeros[0], zeros);
    if (flags) atomicOr(&s.flags, flags);
    if (min_p > 0.f && above) atomicAdd(&s.n_min, above);
}

__device__ __forceinline__ void clear_floats(FloatLds &s)
{
    for (int i = threadIdx.x; i < kSide / 2; i += kRowThreads) {
        ((u32x4 *)s.bins)[i] = u32x4{0, 0, 0, 0};
        ((u32x4 *)s.mass)[2 * i] = ((u32x4 *)s.mass)[2 * i + 1] = u32x4{0, 0, 0, 0};
    }
    if (threadIdx.x < 64) s.powers[threadIdx.x] = exp2((double)threadIdx.x / 64.0);
    clear_choice(s);
}

// The choice out of the bins (thread i's counts and weights are in x) and what stands beside them in s
__device__ __forceinline__ void float_choice(const SampleArgs &a, int r, const RowAsk &ask, const Row<true> &row, Chooser<true> &x, FloatLds &s, char *lds)
{
    const int tid = (int)threadIdx.x;
    Chosen got;
    if (!x.choose(a, r, ask, s.zeros[0], got)) {
        __syncthreads();
        sample_row<true>(a, r, ((WideLds *)lds)->row);
        return;
    }
    if (got.listed) {
        if (tid == 0) a.token[r] = (int)got.nth;
        return;
    }
    // zeros: the nth of either sign, looked for run by run
    uint32_t nth = got.nth;
    for (int i0 = 0; i0 < row.pieces; i0 += kRowThreads) {
        uint32_t bits = 0;
        if (i0 + tid < row.pieces) row.piece(i0 + tid, [&](int index, float z) { bits |= (z == 0.f ? 1u : 0u) << ((index + row.off) & 3); });
        const uint32_t in = (uint32_t)__popc(bits), upto = scan_lanes<true>(in);
        const int lane = tid & 63, wave = tid >> 6;
        __syncthreads();
        if (lane == 63) s.wave_first[wave] = upto;
        __syncthreads();
        const uint32_t wc = s.wave_first[lane & (kRowWaves - 1)], wcs = scan_lanes<false>(wc), here = lane_of(wcs, kRowWaves - 1);
        if (nth < here) {
            const int at = __builtin_amdgcn_readfirstlane(wave);
            const uint32_t before = upto - in + lane_of(wcs, at) - lane_of(wc, at);
            if (nth >= before && nth < before + in) {
                for (uint32_t j = before; j < nth; ++j) bits &= bits - 1;
                a.token[r] = (i0 + tid) * 4 - row.off + __ffs((int)bits) - 1;
            }
            return;
        }
        nth -= here;
    }
}

// slot of thread i's j-th bin
__device__ __forceinline__ int own_slot(int j)
{
    const int tid = (int)threadIdx.x, negative = tid >= kRowThreads / 2;
    return 2 * (negative ? (tid - kRowThreads / 2) * 4 + j : kSide - 1 - tid * 4 - j) + negative;
}

__global__ __launch_bounds__(kRowThreads) void sample_floats_kernel(SampleArgs a)
{
    extern __shared__ __align__(16) char lds[];
    FloatLds &s = ((WideLds *)lds)->choose;
    const int r = blockIdx.x;
    const Row<true> row(a.logits, a.stride, r, a.V);
    const RowAsk ask = row_ask(a, r);
    clear_floats(s);
    __syncthreads();
    float_top(row, 0, row.pieces, s);
    __syncthreads();
    Chooser<true> x{s, row};
    x.m = key_value(s.top);
    if (s.flags || !(x.m > -__builtin_inff()) || !usable(ask.t)) {
        if (threadIdx.x == 0) no_token(a, r);
        return;
    }
    x.inv_t = 1.0 / (double)ask.t;
    __syncthreads();
    float_bins(row, 0, row.pieces, ask.min_p, x, s);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x.c[i] = s.bins[0][own_slot(i)];
        x.unit[i] = s.mass[own_slot(i)];
    }
    float_choice(a, r, ask, row, x, s, lds);
}

// Few rows: cut into parts.  The first kernel finds the parts' largest logits (and clears), the second adds what the parts' bins hold to the row's, the third
// chooses.  Whole numbers are added: in whatever order, the sums are the same.
struct FloatRow {
    uint32_t count[2 * kSide];
    unsigned long long mass[2 * kSide], rare_mass[2];
    uint32_t zeros, flags, n_min, rare[2], unused[3];
    uint32_t top[kMostParts], bad[kMostParts];
    unsigned long long list[2][kRare];
};
static_assert(sizeof(FloatRow) % 16 == 0, "the next row's begins at 16 bytes");

__global__ __launch_bounds__(kRowThreads) void sample_float_tops_kernel(SampleArgs a, int parts)
{
    __shared__ uint32_t tops[kRowWaves], bads;
    const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = (int)threadIdx.x;
    const Row<true> row(a.logits, a.stride, r, a.V);
    FloatRow &f = ((FloatRow *)a.ws)[r];
    const int per = (row.pieces + parts - 1) / parts, from = part * per, to = min(from + per, row.pieces);
    if (tid == 0) bads = 0;
    __syncthreads();
    uint32_t top = 0xffffffffu;
    bool bad = false;
    row.span(from, to, [&](int, float z) {
        bad |= !(z < __builtin_inff());
        top = min(top, order_key(z));
    });
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = min(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if ((tid & 63) == 0) tops[tid >> 6] = top;
    if (bad) bads = 1;
    constexpr int kClear = (int)(offsetof(FloatRow, top) / 16);
    static_assert(offsetof(FloatRow, top) % 16 == 0, "cleared in 16 bytes");
    for (int i = part * kRowThreads + tid; i < kClear; i += parts * kRowThreads) ((u32x4 *)&f)[i] = u32x4{0, 0, 0, 0};
    __syncthreads();
    if (tid == 0) {
        for (int i = 1; i < kRowWaves; ++i) top = min(top, tops[i]);
        f.top[part] = top;
        f.bad[part] = bads;
    }
}

// The largest logit of the row's parts; false: there is no distribution
__device__ __forceinline__ bool row_top(const FloatRow &f, int parts, const RowAsk &ask, Chooser<true> &x)
{
    const int lane = threadIdx.x & 63;
    uint32_t top = lane < parts ? f.top[lane & (kMostParts - 1)] : 0xffffffffu;
    const bool bad = __ballot(lane < parts && f.bad[lane & (kMostParts - 1)]) != 0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = min(top, (uint32_t)__shfl_xor((int)top, o, 64));
    x.m = key_value(top);
    x.inv_t = 1.0 / (double)ask.t;
    return !bad && x.m > -__builtin_inff() && usable(ask.t);
}

__global__ __launch_bounds__(kRowThreads) void sample_float_bins_kernel(SampleArgs a, int parts)
{
    extern __shared__ __align__(16) char lds[];
    FloatLds &s = ((WideLds *)lds)->choose;
    const int r = blockIdx.x / parts, part = blockIdx.x - r * parts, tid = (int)threadIdx.x;
    const Row<true> row(a.logits, a.stride, r, a.V);
    const RowAsk ask = row_ask(a, r);
    FloatRow &f = ((FloatRow *)a.ws)[r];
    const int per = (row.pieces + parts - 1) / parts, from = part * per, to = min(from + per, row.pieces);
    Chooser<true> x{s, row};
    if (!row_top(f, parts, ask, x)) return;
    clear_floats(s);
    __syncthreads();
    float_bins(row, from, to, ask.min_p, x, s);
    __syncthreads();
    for (int i = tid; i < 2 * kSide; i += kRowThreads) {
        const uint32_t n = s.bins[0][i];
        if (n) {
            atomicAdd(&f.count[i], n);
            if (s.mass[i]) atomicAdd(&f.mass[i], s.mass[i]);
        }
    }
    if (tid == 0) {
        if (s.zeros[0]) atomicAdd(&f.zeros, s.zeros[0]);
        if (s.flags) atomicOr(&f.flags, s.flags);
        if (s.n_min) atomicAdd(&f.n_min, s.n_min);
    }
    if (tid < 2) {
        const uint32_t n = s.rare[tid];
        if (n) s.runs[tid] = atomicAdd(&f.rare[tid], n);
        if (s.rare_mass[tid]) atomicAdd(&f.rare_mass[tid], s.rare_mass[tid]);
    }
    __syncthreads();
#pragma unroll
    for (int sign = 0; sign < 2; ++sign)
        if ((uint32_t)tid < min(s.rare[sign], (uint32_t)kRare) && s.runs[sign] + tid < (uint32_t)kRare) f.list[sign][s.runs[sign] + tid] = s.list[sign][tid];
}

__global__ __launch_bounds__(kRowThreads) void sample_float_choose_kernel(SampleArgs a, int parts)
{
    extern __shared__ __align__(16) char lds[];
    FloatLds &s = ((WideLds *)lds)->choose;
    const int r = blockIdx.x, tid = (int)threadIdx.x;
    const Row<true> row(a.logits, a.stride, r, a.V);
    const RowAsk ask = row_ask(a, r);
    const FloatRow &f = ((const FloatRow *)a.ws)[r];
    Chooser<true> x{s, row};
    if (!row_top(f, parts, ask, x)) {
        if (tid == 0) no_token(a, r);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x.c[i] = f.count[own_slot(i)];
        x.unit[i] = f.mass[own_slot(i)];
    }
    static_assert(kRare == kRowThreads, "a thread for each rare value");
    const uint32_t rare[2] = {f.rare[0], f.rare[1]};
    clear_floats(s);
    __syncthreads();
#pragma unroll
    for (int sign = 0; sign < 2; ++sign)
        if ((uint32_t)tid < rare[sign]) s.list[sign][tid] = f.list[sign][tid];
    if (tid == 0) {
        s.zeros[0] = f.zeros;
        s.flags = f.flags;
        s.n_min = f.n_min;
        s.rare[0] = rare[0];
        s.rare[1] = rare[1];
        s.rare_mass[0] = f.rare_mass[0];
        s.rare_mass[1] = f.rare_mass[1];
    }
    __syncthreads();
    float_choice(a, r, ask, row, x, s, lds);
}

// Parts of a row: none where there are rows enough, or little of them.  (Whole / in 8 parts, us: 1 row of 32003 11.7 / 14.0, of 65000 14.0 / 14.3, of 151936 21.5 / 16.9, 64 rows of
// 151936 23.4 / 20.5, 96 rows 23.6 / 23.5; 4 and 16 parts: 1 row 18.6 and 16.7, 64 rows 21.1 and 22.4.)
static int sample_parts(int T, int V)
{
    const int pieces = (V + 14) / 8;        // (a row may begin anywhere in its first piece)
    int parts = T <= 64 && pieces >= 10240 ? 8 : 1;
    if (pieces > 4 * 5 * kRowThreads) parts = max(parts, (pieces + 8 * 512 - 1) / (8 * 512));       // longer than a workgroup takes
    return min(parts, kMostParts);
}

// 32-bit logits: three launches instead of one, and the sums in memory between them.  (One row of 32003 as it is / in 7 parts 25.9 / 22.5 us, 37 rows 28.4 / 35.9; rows of 151936
// as they are / in 8: 1 row 80.7 / 35.4, 64 rows 94.0 / 73.3, 96 rows 94.0 / 89.7.)
static int sample_float_parts(int T, int V) { return T <= 64 && V >= 65536 ? min(min(kMostParts, V / 16384), 512 / T) : 1; }

size_t sample_ws_bytes(int T, int V)        // (of either type)
{
    const int parts = sample_parts(T, V);
    const size_t values = parts > 1 ? (size_t)T * parts * sizeof(PartCounts) : 0, floats = sample_float_parts(T, V) > 1 ? (size_t)T * sizeof(FloatRow) : 0;
    return values > floats ? values : floats;
}

template <int NQ>
static int launch_values(const SampleArgs &a, hipStream_t s)
{
    static LdsLimitOnce once;
    int rc = raise_lds_limit((const void *)sample_values_kernel<NQ>, once, "sample_values_kernel");
    if (rc) return rc;
    sample_values_kernel<NQ><<<dim3((unsigned)a.T), dim3(kRowThreads), sizeof(ValueLds), s>>>(a);
    return check_hip(hipGetLastError(), "sample_values_kernel");
}

template <int NR>
static int launch_choose(const SampleArgs &a, int parts, hipStream_t s)
{
    static LdsLimitOnce once;
    int rc = raise_lds_limit((const void *)sample_choose_kernel<NR>, once, "sample_choose_kernel");
    if (rc) return rc;
    sample_choose_kernel<NR><<<dim3((unsigned)a.T), dim3(kRowThreads), sizeof(ValueLds), s>>>(a, parts);
    return check_hip(hipGetLastError(), "sample_choose_kernel");
}

int launch_sample(const SampleArgs &a, hipStream_t s)
{
    if (a.f32) {
        static LdsLimitOnce once[3];
        const int parts = sample_float_parts(a.T, a.V);
        int rc;
        if (parts > 1) {
            if ((rc = raise_lds_limit((const void *)sample_float_bins_kernel, once[0], "sample_float_bins_kernel")) ||
                (rc = raise_lds_limit((const void *)sample_float_choose_kernel, once[1], "sample_float_choose_kernel")))
                return rc;
            const dim3 grid((unsigned)(a.T * parts)), block(kRowThreads);
            sample_float_tops_kernel<<<grid, block, 0, s>>>(a, parts);
            if ((rc = check_hip(hipGetLastError(), "sample_float_tops_kernel"))) return rc;
            sample_float_bins_kernel<<<grid, block, sizeof(FloatLds), s>>>(a, parts);
            if ((rc = check_hip(hipGetLastError(), "sample_float_bins_kernel"))) return rc;
            sample_float_choose_kernel<<<dim3((unsigned)a.T), block, sizeof(WideLds), s>>>(a, parts);
            return check_hip(hipGetLastError(), "sample_float_choose_kernel");
        }
        if ((rc = raise_lds_limit((const void *)sample_floats_kernel, once[2], "sample_floats_kernel"))) return rc;
        sample_floats_kernel<<<dim3((unsigned)a.T), dim3(kRowThreads), sizeof(WideLds), s>>>(a);
        return check_hip(hipGetLastError(), "sample_floats_kernel");
    }
    const int parts = sample_parts(a.T, a.V), pieces = (a.V + 14) / 8;
    if (parts > 1) {
        if ((int64_t)a.T * parts > 0x7fffffffLL) {
            set_error("qarl_sample: %d rows exceed the grid limit", a.T);
            return QARL_ERR_UNSUPPORTED;
        }
        sample_count_kernel<<<dim3((unsigned)(a.T * parts)), dim3(kCountThreads), 0, s>>>(a, parts);
        int rc = check_hip(hipGetLastError(), "sample_count_kernel");
        if (rc) return rc;
        const int per = (pieces + parts - 1) / parts;
        return per <= 4 * kRowThreads ? launch_choose<4>(a, parts, s) : launch_choose<kRuns>(a, parts, s);     // (1280 pieces a part or more)
    }
    const int quarter = (pieces + 3) / 4;
    if (quarter <= kRowThreads) return launch_values<1>(a, s);
    if (quarter <= 2 * kRowThreads) return launch_values<2>(a, s);
    return launch_values<5>(a, s);
}

}  // namespace qarl
