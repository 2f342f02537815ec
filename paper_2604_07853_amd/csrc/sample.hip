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
// 16-bit logits have few values: 4096 bins hold those of size 2^-8 to 2^8 one by one, so that a count says all of a bin, weights are computed once a value
// and not once a token, and a place in the order is a bin and a number.  (sample_count.. below.)  Rows with others that matter, and 32-bit logits, take the general way.
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
    __device__ __forceinline__ void piece(int i, Fn f) const
    {
        const u32x4 w = base[i];
        const int first = i * kPer - off;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const float z = F32 ? __uint_as_float(w[e & 3]) : __uint_as_float(e & 1 ? w[(e >> 1) & 3] & 0xffff0000u : w[(e >> 1) & 3] << 16);
            if ((unsigned)(first + e) < (unsigned)V) f(first + e, z);
        }
    }
    template <typename Fn>
    __device__ __forceinline__ void all(Fn f) const
    {
        for (int i = threadIdx.x; i < pieces; i += kRowThreads) piece(i, f);
    }
};

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
    // (2^52 added: the sum's last bit is a unit)
    return (unsigned long long)__double_as_longlong(w * kUnit + 4503599627370496.0) & 0xfffffffffffffull;
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

__device__ __forceinline__ void give(const SampleArgs &a, int r, int token, double y, unsigned long long whole, unsigned long long kept)
{
    a.token[r] = token;
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
        const Place p = x.find([goal](uint32_t, unsigned long long w) { return (double)w >= goal; });
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
    const double goal = (ask.u >= 0.f ? (double)ask.u : 0.0) * (double)kept;
    Place p = x.find([goal](uint32_t, unsigned long long w) { return (double)w > goal; });
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
        give(a, r, token, ((double)key_value(p.key) - (double)x.m) * x.inv_t, whole, kept);
    }
}

template <bool F32>
__global__ __launch_bounds__(kRowThreads) void sample_rows_kernel(SampleArgs a)
{
    extern __shared__ __align__(16) char lds[];
    sample_row<F32>(a, blockIdx.x, *(RowLds *)lds);
}

// ---- 16-bit logits by value.  A pattern less kFirst, of which bits 11 to 14 are then zero, names its bin: bit 15 the sign, bits 0 to 10 the size.
constexpr uint32_t kFirst = 118 << 7;       // 2^-9
constexpr double kLowest = 128.0;           // 2^7: sixteen powers of two on
constexpr int kSide = 2048;                 // bins of a sign
constexpr int kRare = 2048;                 // room for values below 2^-9 other than zero (one of 1400 tokens of logits that spread by 2.2)
constexpr uint32_t kNone = 0xff80ff80u;     // two -inf
constexpr int kMostParts = 32;

// Where the bins' counts come from: a workgroup that takes a row by itself counts its quarters apart, two to a word; or parts of a row were counted by workgroups
// of their own.  (The part that a token lies in is searched for it; the others need not be read again.)
struct PartCounts {             // in the workspace, for each part
    uint16_t count[2 * kSide];  // by size, the signs side by side: a part has at most 65535 tokens
    uint32_t zeros, flags, rare, unused;
    uint2 list[kRare / 4];      // index, pattern
};
enum { kBad = 1, kHigh = 2, kLow = 4 };

struct ChooseLds {
    uint32_t bins[2][2 * kSide];
    unsigned long long list[kRare];         // the rare values: what they are sorted by (choose), before that their index and pattern
    unsigned long long wave_mass[kRowWaves], rare_mass[2], rare_sum[kRowWaves];
    uint32_t wave_count[kRowWaves], wave_first[kRowWaves];
    uint32_t rare_count[2], rare_top[2];
    uint32_t rare, zeros, flags, n_min, sorted;
    uint32_t runs[64], part_at[kMostParts + 1];
    Place place[2][kRowWaves], spot;
    uint32_t owner;
};
union ValueLds {
    ChooseLds choose;
    RowLds row;         // for rows that take the general way
};

__device__ __forceinline__ float pattern_value(uint32_t b) { return __uint_as_float(b << 16); }
// place of the bin number `bin` of the order among the counts: sizes rising, the signs side by side
__device__ __forceinline__ int bin_slot(int bin) { return bin < kSide ? 2 * (kSide - 1 - bin) : 2 * (bin - kSide) + 1; }
__device__ __forceinline__ uint32_t bin_pattern(int bin) { return bin < kSide ? kFirst + (uint32_t)(kSide - 1 - bin) : 0x8000u + kFirst + (uint32_t)(bin - kSide); }

// Two values into the bins (`bump` to be added to their counts), or to what is kept of others
__device__ __forceinline__ void count_pair(uint32_t w, int index, uint32_t *bins, uint32_t bump, ChooseLds &s, uint32_t &zeros, uint32_t &flags)
{
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
    const u16x2 r = __builtin_bit_cast(u16x2, w) - (u16x2){(uint16_t)kFirst, (uint16_t)kFirst};
    const uint32_t slot = __builtin_bit_cast(uint32_t, (u16x2)(r << 1)) | __builtin_bit_cast(uint32_t, (u16x2)(r >> 15));
    const uint32_t rw = __builtin_bit_cast(uint32_t, r);
    if ((rw & 0x78007800u) == 0) {
        atomicAdd((uint32_t *)((char *)bins + ((slot << 2) & 0x3fffcu)), bump);
        atomicAdd((uint32_t *)((char *)bins + ((slot >> 14) & 0x3fffcu)), bump);
        return;
    }
    if (w == kNone) return;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t b = e ? w >> 16 : w & 0xffffu, rb = e ? rw >> 16 : rw & 0xffffu, size = b & 0x7fffu;
        if ((rb & 0x7800u) == 0) {
            atomicAdd(bins + (e ? slot >> 16 : slot & 0xffffu), bump);
        } else if (size == 0) {
            ++zeros;
        } else if (size < kFirst) {
            const uint32_t at = atomicAdd(&s.rare, 1u);
            if (at < (uint32_t)kRare) s.list[at] = (unsigned long long)b << 32 | (uint32_t)(index + e);
        } else if (b != 0xff80u) {
            flags |= size >= 0x7f80u ? kBad : b & 0x8000u ? kLow : kHigh;
        }
    }
}
// Eight values; those outside the row become -inf
__device__ __forceinline__ void count_piece(u32x4 w, int first, int V, uint32_t *bins, uint32_t bump, ChooseLds &s, uint32_t &zeros, uint32_t &flags)
{
    if (first < 0 || first + 8 > V) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((unsigned)(first + e) >= (unsigned)V) w[e >> 1] = e & 1 ? (w[e >> 1] & 0xffffu) | (kNone & 0xffff0000u) : (w[e >> 1] & 0xffff0000u) | (kNone & 0xffffu);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) count_pair(w[e], first + 2 * e, bins, bump, s, zeros, flags);
}

struct Chosen {
    uint32_t pattern;       // the token's value
    uint32_t nth;           // of the tokens with that value; of a rare one: its index
    bool rare, none;
    double y;
    unsigned long long whole, kept;
};

// What the counts of a row say.  Thread i holds bins 4 i .. 4 i + 3 of the order: positive values falling, then negative ones; the rare ones and zero stand between.
struct Chooser {
    static constexpr int kEach = 2 * kSide / kRowThreads;
    ChooseLds &s;
    uint32_t c[kEach], cb;
    unsigned long long unit[kEach], mb;
    uint32_t special[3];                        // tokens of the rare positive values, of zero, of the rare negative ones
    unsigned long long special_mass[3], zero_unit;
    float m;
    double inv_t;
    int calls;

    __device__ __forceinline__ unsigned long long weigh(float z, double &w) const { return weight_of(((double)z - (double)m) * inv_t, w); }

    // The place among the rare values of a sign, each a bin of its own.  They are sorted the first time that one is asked for: by value falling, then index.
    // (`from`, `count`: of that sign; the result in s.spot, its index in s.owner.  A function of its own: it is seldom called, and costs the others registers.)
    template <typename Fn>
    __device__ static __attribute__((noinline)) void among_rare(ChooseLds &s, uint32_t from, uint32_t count, uint32_t before, unsigned long long mass, float m, double inv_t, Fn pass)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const uint32_t n = s.rare;
        __syncthreads();
        if (!s.sorted) {
            uint32_t size = 2;
            while (size < n) size *= 2;
            for (uint32_t i = threadIdx.x; i < size; i += kRowThreads) {
                unsigned long long k = ~0ull;
                if (i < n) {
                    const uint32_t b = (uint32_t)(s.list[i] >> 32);     // (patterns of positive values turned round: falling)
                    k = (unsigned long long)(b >> 15 ? b : 0x7fffu - b) << 32 | (uint32_t)s.list[i];
                }
                s.list[i] = k;
            }
            for (uint32_t k = 2; k <= size; k *= 2) {
                for (uint32_t j = k / 2; j > 0; j /= 2) {
                    __syncthreads();
                    for (uint32_t t = threadIdx.x; t < size / 2; t += kRowThreads) {
                        const uint32_t a = 2 * t - (t & (j - 1)), b = a + j;
                        const unsigned long long x = s.list[a], y = s.list[b];
                        if ((x > y) == ((a & k) == 0)) {
                            s.list[a] = y;
                            s.list[b] = x;
                        }
                    }
                }
            }
            __syncthreads();
            if (threadIdx.x == 0) s.sorted = 1;
        }
        // positive ones stand in front; thread i takes entries 2 i and 2 i + 1 of its sign
        unsigned long long u[2] = {0, 0}, key[2] = {0, 0};
        double w;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t i = 2 * threadIdx.x + e;
            if (i < count) {
                key[e] = s.list[from + i];
                const uint32_t b = (uint32_t)(key[e] >> 32);
                key[e] = (unsigned long long)(b >> 15 ? b : 0x7fffu - b) << 32 | (uint32_t)key[e];
                u[e] = weight_of(((double)pattern_value((uint32_t)(key[e] >> 32)) - (double)m) * inv_t, w);
            }
        }
        unsigned long long wi = u[0] + u[1];
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const unsigned long long up = __shfl_up(wi, o, 64);
            if (lane >= o) wi += up;
        }
        if (lane == 63) s.rare_sum[wave] = wi;
        __syncthreads();
        mass += wi - u[0] - u[1];
        for (int i = 0; i < wave; ++i) mass += s.rare_sum[i];
        before += 2 * threadIdx.x;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const uint32_t i = 2 * threadIdx.x + e;
            // the first that passes: what stands in front of it does not
            if (i < count && pass(before + 1, mass + u[e]) && (i == 0 || !pass(before, mass))) {
                s.spot = Place{(uint32_t)(key[e] >> 32), before, 1, mass, u[e], true};
                s.owner = (uint32_t)key[e];
            }
            before += 1;
            mass += u[e];
        }
        __syncthreads();
    }

    template <typename Fn>
    __device__ __forceinline__ Place find(Fn pass, bool &rare)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        Place *const places = s.place[calls++ & 1];     // (the other half may still be read)
        Place mine = {};
        uint32_t before = cb;
        unsigned long long mass = mb;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (!mine.there && c[i] && pass(before + c[i], mass + c[i] * unit[i])) mine = Place{bin_pattern(threadIdx.x * kEach + i), before, c[i], mass, unit[i], true};
            before += c[i];
            mass += c[i] * unit[i];
        }
        const unsigned long long hit = __ballot(mine.there);
        if (lane == (hit ? __ffsll((long long)hit) - 1 : 0)) places[wave] = mine;
        __syncthreads();
        rare = false;
#pragma unroll 1
        for (int i = 0; i < kRowWaves; ++i) {
            if (i == kRowWaves / 2) {       // between the signs
                uint32_t b = 0;
                unsigned long long w = 0;
                for (int j = 0; j < kRowWaves / 2; ++j) {
                    b += s.wave_count[j];
                    w += s.wave_mass[j];
                }
                for (int j = 0; j < 3; ++j) {
                    if (special[j] && pass(b + special[j], w + special_mass[j])) {
                        if (j == 1) return Place{0, b, special[1], w, zero_unit, true};
                        rare = true;
                        among_rare(s, j ? special[0] : 0, special[j], b, w, m, inv_t, pass);
                        return s.spot;
                    }
                    b += special[j];
                    w += special_mass[j];
                }
            }
            if (places[i].there) return places[i];
        }
        return Place{};
    }

    // False where the row has to take the general way
    __device__ __forceinline__ bool choose(const RowAsk &ask, Chosen &out)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        calls = 0;
        const uint32_t n_rare = min(s.rare, (uint32_t)kRare);
        // ---- the largest value
        int first = -1;
#pragma unroll
        for (int i = kEach - 1; i >= 0; --i)
            if (c[i]) first = threadIdx.x * kEach + i;
        const unsigned long long some = __ballot(first >= 0);
        if (lane == (some ? __ffsll((long long)some) - 1 : 0)) s.wave_first[wave] = (uint32_t)first;
        for (uint32_t i = threadIdx.x; i < n_rare; i += kRowThreads) {
            const uint32_t b = (uint32_t)(s.list[i] >> 32);
            if (b >> 15) atomicMin(&s.rare_top[1], b);
            else atomicMax(&s.rare_top[0], b);
            atomicAdd(&s.rare_count[b >> 15], 1u);
        }
        __syncthreads();
        out.none = true;
        if ((s.flags & kBad) || !usable(ask.t)) return true;
        if ((s.flags & kHigh) || s.rare > (uint32_t)kRare) return false;
        special[0] = s.rare_count[0];
        special[1] = s.zeros;
        special[2] = s.rare_count[1];
        uint32_t top = 0xffffffffu;
        for (int i = 0; i < kRowWaves && top == 0xffffffffu; ++i) {
            if (i == kRowWaves / 2) {
                if (special[0]) top = s.rare_top[0];
                else if (special[1]) top = 0;
                else if (special[2]) top = s.rare_top[1];
                if (top != 0xffffffffu) break;
            }
            if ((int)s.wave_first[i] >= 0) top = bin_pattern((int)s.wave_first[i]);
        }
        if (top == 0xffffffffu) return !(s.flags & kLow);       // (only -inf: no token)
        m = pattern_value(top);
        inv_t = 1.0 / (double)ask.t;
        if ((s.flags & kLow) && ((double)m + kLowest) * inv_t < 31.0) return false;     // those of -128 and less weigh a unit or more
        // ---- weights
        uint32_t csum = 0, above = 0;
        unsigned long long wsum = 0;
        double w;
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            unit[i] = 0;
            if (c[i]) {
                unit[i] = weigh(pattern_value(bin_pattern(threadIdx.x * kEach + i)), w);
                if (w >= (double)ask.min_p) above += c[i];
            }
            csum += c[i];
            wsum += c[i] * unit[i];
        }
        for (uint32_t i = threadIdx.x; i < n_rare; i += kRowThreads) {
            const uint32_t b = (uint32_t)(s.list[i] >> 32);
            const unsigned long long units = weigh(pattern_value(b), w);
            if (units) atomicAdd(&s.rare_mass[b >> 15], units);
            above += w >= (double)ask.min_p;
        }
        zero_unit = weigh(0.f, w);
        if (threadIdx.x == 0 && w >= (double)ask.min_p) above += special[1];
        if (ask.min_p > 0.f && above) atomicAdd(&s.n_min, above);
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
        __syncthreads();
        special_mass[0] = s.rare_mass[0];
        special_mass[1] = special[1] * zero_unit;
        special_mass[2] = s.rare_mass[1];
        cb = ci - csum;
        mb = wi - wsum;
        uint32_t n = special[0] + special[1] + special[2];
        unsigned long long whole = special_mass[0] + special_mass[1] + special_mass[2];
        if (wave >= kRowWaves / 2) {
            cb += n;
            mb += whole;
        }
#pragma unroll 1
        for (int i = 0; i < kRowWaves; ++i) {
            if (i < wave) {
                cb += s.wave_count[i];
                mb += s.wave_mass[i];
            }
            n += s.wave_count[i];
            whole += s.wave_mass[i];
        }
        // ---- what is kept, and the token
        unsigned long long kept = whole;
        bool rare;
        const auto first_tokens = [&](uint32_t k) {
            const Place p = find([k](uint32_t x, unsigned long long) { return x >= k; }, rare);
            n = k;
            kept = p.mass + (k - p.before) * p.each;
        };
        if (ask.k > 0 && (uint32_t)ask.k < n) first_tokens((uint32_t)ask.k);
        if (ask.top_p < 1.f && n > 1) {
            const double goal = (double)fmaxf(ask.top_p, 0.f) * (double)kept;
            const Place p = find([goal](uint32_t, unsigned long long x) { return (double)x >= goal; }, rare);
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
        const double goal = (ask.u >= 0.f ? (double)ask.u : 0.0) * (double)kept;
        Place p = find([goal](uint32_t, unsigned long long x) { return (double)x > goal; }, rare);
        if (p.there && p.before < n) {
            out.nth = p.each ? (uint32_t)fmin(fmax(floor((goal - (double)p.mass) / (double)p.each), 0.0), (double)(p.equal - 1)) : 0u;
            out.nth = min(out.nth, n - 1 - p.before);
        } else {        // the last one of any weight
            const unsigned long long all = kept;
            p = find([all](uint32_t, unsigned long long x) { return x >= all; }, rare);
            out.nth = (uint32_t)((kept - p.mass - 1) / p.each);
        }
        if (rare) out.nth = s.owner;
        out.pattern = p.key;
        out.rare = rare;
        out.none = false;
        out.y = ((double)pattern_value(p.key) - (double)m) * inv_t;
        out.whole = whole;
        out.kept = kept;
        return true;
    }
};

__device__ __forceinline__ void clear_choice(ChooseLds &s)
{
    if (threadIdx.x < 64) s.runs[threadIdx.x] = 0;
    if (threadIdx.x == 0) {
        s.rare = s.zeros = s.flags = s.n_min = s.sorted = 0;
        s.rare_count[0] = s.rare_count[1] = 0;
        s.rare_mass[0] = s.rare_mass[1] = 0;
        s.rare_top[0] = 0;
        s.rare_top[1] = 0xffffffffu;
    }
}

// The index of the nth token with that pattern among pieces [from, to), and the answer.  First the run of kRowThreads pieces, then the thread, then the element.
__device__ __forceinline__ void answer(const SampleArgs &a, int r, const Row<false> &row, int from, int to, uint32_t nth, const Chosen &got, ChooseLds &s)
{
    const uint32_t keep = got.pattern ? 0xffffu : 0x7fffu;      // (zeros of either sign)
    const auto matches = [&](u32x4 w, int first) {
        uint32_t n = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            n |= (((e & 1 ? w[e >> 1] >> 16 : w[e >> 1]) & keep) == got.pattern && (unsigned)(first + e) < (unsigned)row.V ? 1u : 0u) << e;
        return n;
    };
    for (int i = from + (int)threadIdx.x, run = 0; i < to; i += kRowThreads, ++run) {
        const uint32_t n = __popc(matches(row.base[i], i * 8 - row.off));
        if (n) atomicAdd(&s.runs[run], n);
    }
    __syncthreads();
    int run = 0;
    while (run < 63 && nth >= s.runs[run]) nth -= s.runs[run++];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, i = from + run * kRowThreads + (int)threadIdx.x;
    const uint32_t bits = i < to ? matches(row.base[i], i * 8 - row.off) : 0u, in = __popc(bits);
    uint32_t upto = in;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(upto, o, 64);
        if (lane >= o) upto += up;
    }
    if (lane == 63) s.wave_first[wave] = upto;
    __syncthreads();
    uint32_t before = upto - in;
    for (int j = 0; j < wave; ++j) before += s.wave_first[j];
    if (nth >= before && nth < before + in) {
        uint32_t left = bits;
        for (uint32_t j = before; j < nth; ++j) left &= left - 1;
        give(a, r, i * 8 - row.off + __ffs((int)left) - 1, got.y, got.whole, got.kept);
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
    const auto load = [&](int q) {
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int in = i * kRowThreads + tid;
            w[q & 1][i] = u32x4{kNone, kNone, kNone, kNone};
            if (in < quarter && q * quarter + in < row.pieces) w[q & 1][i] = row.base[q * quarter + in];
        }
    };
    load(0);
    for (int i = tid; i < kSide; i += kRowThreads) ((u32x4 *)s.bins)[i] = u32x4{0, 0, 0, 0};
    clear_choice(s);
    __syncthreads();
    uint32_t zeros = 0, flags = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (q < 3) load(q + 1);
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const int in = i * kRowThreads + tid;
            if (in < quarter) count_piece(w[q & 1][i], (q * quarter + in) * 8 - row.off, a.V, s.bins[q >> 1], q & 1 ? 65536u : 1u, s, zeros, flags);
        }
    }
    if (zeros) atomicAdd(&s.zeros, zeros);
    if (flags) atomicOr(&s.flags, flags);
    __syncthreads();
    Chooser x{s};
#pragma unroll
    for (int i = 0; i < Chooser::kEach; ++i) {
        const int at = bin_slot(tid * Chooser::kEach + i);
        const uint32_t lo = s.bins[0][at], hi = s.bins[1][at];
        x.c[i] = (lo & 0xffffu) + (lo >> 16) + (hi & 0xffffu) + (hi >> 16);
    }
    Chosen got;
    if (!x.choose(row_ask(a, r), got)) {
        __syncthreads();
        sample_row<false>(a, r, ((ValueLds *)lds)->row);
        return;
    }
    if (got.none || got.rare) {
        if (tid == 0) {
            if (got.none) no_token(a, r);
            else give(a, r, (int)got.nth, got.y, got.whole, got.kept);
        }
        return;
    }
    uint32_t nth = got.nth;
    int q = 0;
    if (got.pattern) {      // (zeros are not counted by quarters: all of the row is searched for them)
        const uint32_t size = (got.pattern & 0x7fffu) - kFirst, at = 2 * size + (got.pattern >> 15);
        const uint32_t lo = s.bins[0][at], hi = s.bins[1][at];
        const uint32_t n[3] = {lo & 0xffffu, lo >> 16, hi & 0xffffu};
        while (q < 3 && nth >= n[q]) nth -= n[q++];
        answer(a, r, row, q * quarter, min((q + 1) * quarter, row.pieces), nth, got, s);
    } else {
        answer(a, r, row, 0, row.pieces, nth, got, s);
    }
}

size_t sample_ws_bytes(int, int) { return 0; }

template <int NQ>
static int launch_values(const SampleArgs &a, hipStream_t s)
{
    static LdsLimitOnce once;
    int rc = raise_lds_limit((const void *)sample_values_kernel<NQ>, once, "sample_values_kernel");
    if (rc) return rc;
    sample_values_kernel<NQ><<<dim3((unsigned)a.T), dim3(kRowThreads), sizeof(ValueLds), s>>>(a);
    return check_hip(hipGetLastError(), "sample_values_kernel");
}

int launch_sample(const SampleArgs &a, hipStream_t s)
{
    const int quarter = ((a.V + 7 + 7) / 8 + 3) / 4;      // (a row may begin anywhere in its first piece)
    if (!a.f32 && quarter <= kRowThreads) return launch_values<1>(a, s);
    if (!a.f32 && quarter <= 2 * kRowThreads) return launch_values<2>(a, s);
    if (!a.f32 && quarter <= 5 * kRowThreads) return launch_values<5>(a, s);
    static LdsLimitOnce once[2];
    int rc = raise_lds_limit(a.f32 ? (const void *)sample_rows_kernel<true> : (const void *)sample_rows_kernel<false>, once[a.f32 ? 1 : 0], "sample_rows_kernel");
    if (rc) return rc;
    if (a.f32) sample_rows_kernel<true><<<dim3((unsigned)a.T), dim3(kRowThreads), sizeof(RowLds), s>>>(a);
    else sample_rows_kernel<false><<<dim3((unsigned)a.T), dim3(kRowThreads), sizeof(RowLds), s>>>(a);
    return check_hip(hipGetLastError(), "sample_rows_kernel");
}

}  // namespace qarl
