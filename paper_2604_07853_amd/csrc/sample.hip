// The next token of each row of logits, by temperature, top-k, top-p, min-p and one given random number.
//
// Tokens stand in the order of their logits, equal ones by index; token i weighs w_i = e^((z_i - m) / t), m the largest logit.  All three truncations leave a
// beginning of that order, so all that is asked of a row are places in it: the first k tokens, the shortest beginning that holds p of their weight,
// the tokens of weight min_p and more, and the token at which the kept weights reach u times their sum.  A place is found without sorting: by the counts
// and weights of 4096 bins of the order, then of 4096 parts of the bin that it lies in, until that is a single value.
//
// Sums decide between tokens, and a sum that is off by one part in 10^7 takes another token in one of a thousand rows of a wide distribution.  Weights
// are therefore computed in 64 bits and summed as integers, in units of 2^-43: whatever the order of the additions, a row's token is the same.
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
        return (unsigned long long)__double2ll_rn(exp(((double)z - (double)m) * inv_t) * kUnit);
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

template <bool F32>
__global__ __launch_bounds__(kRowThreads) void sample_rows_kernel(SampleArgs a)
{
    extern __shared__ __align__(16) char lds[];
    RowLds &s = *(RowLds *)lds;
    const int r = blockIdx.x;
    RowSampler<F32> x{Row<F32>(a.logits, a.stride, r, a.V), s};
    float t = a.temperature ? a.temperature[r] : 1.f;
    const bool greedy = t == 0.f;
    if (greedy) t = 1.f;
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
    if (s.flags || !(x.m > -__builtin_inff()) || !(t > 0.f && t < __builtin_inff())) {
        if (threadIdx.x == 0) {
            a.token[r] = -1;
            if (a.logprob) a.logprob[r] = __builtin_nanf("");
            if (a.kept_logprob) a.kept_logprob[r] = __builtin_nanf("");
        }
        return;
    }
    x.inv_t = 1.0 / (double)t;
    x.bin_scale = fminf((float)(kBins - 1) / (kWindow * t), 1e30f);
    // ---- counts and weights of the bins; the tokens that min-p leaves
    float min_p = a.min_p ? a.min_p[r] : 0.f;
    if (!(min_p > 0.f)) min_p = 0.f;
    uint32_t n_min = 0;
    if (threadIdx.x == 0) s.flags = 0;
    __syncthreads();
    x.row.all([&](int, float z) {
        if (z > -__builtin_inff()) {
            const double w = exp(((double)z - (double)x.m) * x.inv_t);
            const int b = x.bin(z);
            atomicAdd(&s.first.count[b], 1u);
            atomicAdd(&s.first.mass[b], (unsigned long long)__double2ll_rn(w * kUnit));
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
    const int k = greedy ? 1 : a.top_k ? a.top_k[r] : 0;
    if (k > 0 && (uint32_t)k < n) first_tokens((uint32_t)k);
    const float top_p = a.top_p ? a.top_p[r] : 1.f;
    if (top_p < 1.f && n > 1) {
        const double goal = (double)fmaxf(top_p, 0.f) * (double)kept;
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
    const float u = a.u[r];
    const double goal = (u >= 0.f ? (double)u : 0.0) * (double)kept;
    Place p = x.find([goal](uint32_t, unsigned long long w) { return (double)w > goal; });
    uint32_t nth = 0;
    if (p.there && p.before < n) {
        nth = p.each ? (uint32_t)fmin(fmax(floor((goal - (double)p.mass) / (double)p.each), 0.0), (double)(p.equal - 1)) : 0u;
        nth = min(nth, n - 1 - p.before);
    } else {
        const uint32_t last = n;
        p = x.find([last](uint32_t c, unsigned long long) { return c >= last; });
        nth = n - 1 - p.before;
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
        const double y = ((double)key_value(p.key) - (double)x.m) * x.inv_t;
        if (a.logprob) a.logprob[r] = (float)(y - log((double)whole / kUnit));
        if (a.kept_logprob) a.kept_logprob[r] = (float)(y - log((double)kept / kUnit));
    }
}

size_t sample_ws_bytes(int, int) { return 0; }

int launch_sample(const SampleArgs &a, hipStream_t s)
{
    static LdsLimitOnce once[2];
    int rc = raise_lds_limit(a.f32 ? (const void *)sample_rows_kernel<true> : (const void *)sample_rows_kernel<false>, once[a.f32 ? 1 : 0], "sample_rows_kernel");
    if (rc) return rc;
    if (a.f32) sample_rows_kernel<true><<<dim3((unsigned)a.T), dim3(kRowThreads), sizeof(RowLds), s>>>(a);
    else sample_rows_kernel<false><<<dim3((unsigned)a.T), dim3(kRowThreads), sizeof(RowLds), s>>>(a);
    return check_hip(hipGetLastError(), "sample_rows_kernel");
}

}  // namespace qarl
