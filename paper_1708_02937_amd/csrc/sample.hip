// The next token of each row of logits.
//
//   x_i = (max l - l_i) / temperature,  p_i = exp(-x_i)
//   K = the top_k tokens with the largest logits (equal ones by index),  P = the shortest run of K in that order whose mass is
//   top_p of K's or more,  M = the tokens with p_i >= min_p;  all three are beginnings of one order, and so is what is kept
//   token = the first index at which the mass of the kept tokens up to it exceeds u times the mass of all of them
//
// Which token it is goes by sums in 64 bits: 32 do not tell the tokens of a large vocabulary apart.  Nothing is sorted.  A
// row's tokens are counted in buckets of x, a 16th wide, with their mass as whole numbers, so that the order of the additions
// does not matter; the buckets tell where the order ends, within a bucket or a few, and only the tokens of those, the list, are
// looked at one by one.  Buckets before them are kept whole.
//
// A token is a number: its logit's place in the order of floats above the complement of its index, so that a larger one
// comes first and no two are equal.
//
// A bucket's masses are in units of exp(-b / 16) 2^-shift: e^-d for 0 <= d < 1/16 is a polynomial, of degree 7 where it is rounded to
// such a unit and 8 elsewhere (the next terms are 6e-15 and 4e-17), and the sum of a bucket is as exact as its values.  The last bucket is x >= 63.9: its tokens count, but their mass,
// below 2e-28 of the first token's each, is 0.
#include <algorithm>

#include "blocks8.h"
#include "common.h"
#include "lanes.h"
#include "shared_memory.h"

namespace sdnn {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kTile = kThreads * 8;  // tokens that a workgroup looks at in turn
constexpr int kBuckets = 1024, kPerNat = 16, kEach = kBuckets / kThreads;
constexpr int kList = 4096;          // tokens of the list that fit LDS; of a longer one they are looked for in the row each time
constexpr int kRanked = kThreads;    // up to so many are ranked by counting
constexpr int kCountOnly = 1024;     // up to so many tokens kept by top_k, masses are not summed over the row

// The order of logits as numbers above 0; 0 for one that cannot be taken (-inf, NaN).
__device__ __forceinline__ uint32_t key_of(float l) {
    if (!(l > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(l + 0.0f);  // -0 is 0
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of_key(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint64_t token_of(uint32_t key, int64_t index) {
    return (uint64_t)key << 32 | (uint32_t)~(uint32_t)index;
}
__device__ __forceinline__ int64_t index_of(uint64_t token) { return (uint32_t)~(uint32_t)token; }

// Settings of a row, and x of its logits.
struct Row {
    double u, top_p, inverse;  // of the temperature
    double most_x;             // x of min_p
    int64_t top_k;
    float top;  // largest logit
    bool masses;

    __device__ __forceinline__ double x(uint32_t key) const {
        const float l = logit_of_key(key);
        return l == top ? 0.0 : ((double)top - (double)l) * inverse;
    }
};

__device__ __forceinline__ bool is_greedy(const SampleArgs &a, int64_t at) {
    return a.temperature && !(a.temperature[at] > 0.0f);
}

__device__ __forceinline__ Row row_of(const SampleArgs &a, int64_t at) {
    Row r;
    double temperature = a.temperature ? (double)a.temperature[at] : 1.0;
    const double min_p = a.min_p ? (double)a.min_p[at] : 0.0;
    r.u = a.uniform[at];
    r.top_k = a.top_k ? a.top_k[at] : 0;
    r.top_p = a.top_p ? (double)a.top_p[at] : 1.0;
    if (r.top_p < 0.0) r.top_p = 0.0;
    if (temperature == (double)INFINITY) temperature = 1e300;  // every token alike
    r.inverse = 1.0 / temperature;
    r.most_x = min_p > 0.0 ? -log(fmin(min_p, 1.0)) : (double)INFINITY;
    r.masses = !(r.top_k > 0 && r.top_k <= kCountOnly);
    return r;
}

// Buckets of a range of x.  The whole row's are a 16th wide; the list's tokens are counted again in narrower ones.
struct Level {
    double start, width, inverse;  // of the width
    __device__ __forceinline__ int bucket(double x) const {
        return (int)fmin(fmax((x - start) * inverse, 0.0), (double)(kBuckets - 1));
    }
    __device__ __forceinline__ double from(int b) const { return fma((double)b, width, start); }
};
__device__ __forceinline__ Level row_level() { return {0.0, 1.0 / kPerNat, (double)kPerNat}; }
__device__ __forceinline__ Level list_level(int lo, int hi) {
    const double width = (double)(hi - lo + 1) / (kPerNat * kBuckets);
    return {(double)lo / kPerNat, width, 1.0 / width};
}

// e^-d, 0 <= d <= 1/16.
__device__ __forceinline__ double exp_small(double d) {
    double e = 1.0 / 40320.0;
    e = fma(-d, e, 1.0 / 5040.0), e = fma(-d, e, 1.0 / 720.0), e = fma(-d, e, 1.0 / 120.0), e = fma(-d, e, 1.0 / 24.0);
    e = fma(-d, e, 1.0 / 6.0), e = fma(-d, e, 0.5), e = fma(-d, e, 1.0);
    return fma(-d, e, 1.0);
}

// e^-(d / 16), 0 <= d <= 1, to 6e-15, a fifth of what rounding to 2^-44 takes from it.
__device__ __forceinline__ double exp_sixteenth(double d) {
    double e = -1.0 / (5040.0 * 268435456.0);
    e = fma(d, e, 1.0 / (720.0 * 16777216.0)), e = fma(d, e, -1.0 / (120.0 * 1048576.0));
    e = fma(d, e, 1.0 / (24.0 * 65536.0)), e = fma(d, e, -1.0 / (6.0 * 4096.0)), e = fma(d, e, 1.0 / 512.0);
    return fma(d, fma(d, e, -1.0 / 16.0), 1.0);
}

// Past this tokens have no mass: the row's last bucket.
__device__ __forceinline__ bool weighs(double x) { return x * kPerNat < (double)(kBuckets - 1); }

// e^-x from e^-(b / 16) of the bucket b that x is in.
__device__ __forceinline__ double mass(double x, const double *table) {
    if (!weighs(x)) return 0.0;
    const int b = (int)(x * kPerNat);
    return table[b] * exp_small(x - (double)b / kPerNat);
}

// Its last place is 2^-shift.
__device__ __forceinline__ double magic_of(int shift) { return __hiloint2double((1023 + 52 - shift) << 20, 0); }

// The mass of x in the unit of its bucket, which starts at `from`: a whole number of 2^-shift.
__device__ __forceinline__ uint64_t whole_mass(double x, double from, int shift) {
    if (!weighs(x)) return 0;
    return (uint64_t)__double_as_longlong(exp_small(x - from) + magic_of(shift)) & ((1ull << 52) - 1);
}

struct Keys {
    uint32_t first, end;  // keys from this on and before that
};

// What the buckets tell of a row.
struct Plan {
    int64_t k;       // tokens that top_k leaves
    int64_t before;  // tokens of the buckets before lo, and their mass
    double above;
    double all;         // the row's mass (0: not known, and without a cut by top_k the list goes to the row's end)
    int lo, hi;         // buckets of the list (hi < lo: none); those before are kept whole, those after not at all
    bool cut_k, cut_p;  // whether there is anything to cut within the list
    bool settled;       // the row has been answered
    uint32_t bound;     // the list is of keys from this on, by the groups; 0: by the buckets
    float top;
    Keys keys;          // the list's
};

struct SampleSpace {
    uint64_t *best;    // rows x chunks: the first token
    uint64_t *masses;  // rows x buckets
    uint64_t *parts;   // rows x chunks x buckets: the chunk's masses
    uint64_t *list;    // rows x chunks x chunk / 8 tokens
    double *whole;     // rows x chunks: mass of the chunk's tokens in buckets that are kept whole
    Plan *plan;        // rows
    uint32_t *counts;  // rows x buckets
    uint32_t *listed;  // rows x chunks: tokens in the list's buckets
    uint32_t *done;    // rows: chunks that are counted
};

// Tokens of a chunk: whole tiles, so that a call has about 1024 workgroups.
int64_t tiles_of(int64_t vocab) { return (vocab + kTile - 1) / kTile; }
int64_t chunk_of(int64_t rows, int64_t vocab) {
    const int64_t each = rows < 1024 ? 1024 / rows : 1;
    return (tiles_of(vocab) + each - 1) / each * kTile;
}

// Of bounds that grow with the rows, so that the space for the most rows holds any call of fewer.
size_t sample_sizes(int64_t rows, int64_t vocab, void *at, SampleSpace *ws) {
    const int64_t tiles = tiles_of(vocab), chunk = chunk_of(rows, vocab);
    const size_t most = rows < 1024 ? 1024 : rows, chunks = (size_t)(rows < (int64_t)most / tiles ? rows * tiles : most);
    char *p = (char *)at;
    auto take = [&](size_t bytes) {
        char *const q = p;
        p += align_up(bytes);
        return q;
    };
    SampleSpace s;
    s.best = (uint64_t *)take(chunks * 8);
    s.masses = (uint64_t *)take(rows * kBuckets * 8);
    s.parts = (uint64_t *)take(chunks * kBuckets * 8);
    s.list = (uint64_t *)take((size_t)rows * (tiles * kTile + chunk - kTile) / 8 * 8);
    s.whole = (double *)take(chunks * 8);
    s.plan = (Plan *)take(rows * sizeof(Plan));
    s.counts = (uint32_t *)take(rows * kBuckets * 4);
    s.listed = (uint32_t *)take(chunks * 4);
    s.done = (uint32_t *)take(rows * 4);
    if (ws) *ws = s;
    return (size_t)(p - (char *)at);
}

// ------------------------------------------------------------------------------------------------ over a workgroup
struct Hist {
    uint64_t masses[kBuckets];
    uint32_t counts[kBuckets];
};

constexpr int kBins = 256;  // of one of the eight levels of a selection by the bits of a token

struct Common {
    union {
        Hist hist;
        struct {
            uint64_t masses[kBins];
            uint32_t counts[kBins];
        } bins;
        struct {
            uint64_t token[kRanked];
            double mass[kRanked];
        } sorted;
        uint16_t upto[kList];  // of the list's tokens up to there: how many are kept and have a mass
    };
    double part[kWaves];
    uint64_t upart[kWaves];
    int64_t ipart[kWaves];
    int64_t found[2];
    double value[2];
};

struct Shared : Common {
    uint64_t list[kList];  // in order of the indices; later the mass of what is kept of it up to there
    uint64_t few[kRanked];
    double table[kBuckets];  // e^-(b / 16)
    uint32_t offset[kThreads + 1];  // of the chunks' parts of the list
};

__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t *part) {
    v = wave_max_last(v);
    __syncthreads();
    if (threadIdx.x % 64 == 63) part[threadIdx.x / 64] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kWaves; w++) v = max64(v, part[w]);
    return v;
}

// The sum of the threads' values up to this one's, and of all, in one order.
template <typename V>
__device__ __forceinline__ V block_upto(V v, V *part, V &all) {
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    v = wave_upto(v);
    __syncthreads();
    if (lane == 63) part[wave] = v;
    __syncthreads();
    all = V(0);
    V before = V(0);
    for (int w = 0; w < kWaves; w++) {
        if (w == wave) before = all;
        all += part[w];
    }
    return before + v;
}

template <typename V>
__device__ __forceinline__ V block_sum(V v, V *part) {
    V all;
    block_upto(v, part, all);
    return all;
}

// The first thread with `hit`, or, where none has it, the last with `some`; -1 where none has either.
__device__ __forceinline__ int elect(bool hit, bool some, Common &sh) {
    const uint64_t best = block_max(hit ? (uint64_t)(kThreads - threadIdx.x) << 32 : some ? threadIdx.x + 1 : 0, sh.upart);
    return best >> 32 ? kThreads - (int)(best >> 32) : (int)best - 1;
}

// f(logits, first index) for the tokens [begin, end), eight at a time (NaN past the end), the next ones on their way meanwhile.
// next: this thread's first ones, by first_logits.
template <typename T>
__device__ __forceinline__ void logits8(const T *row, int64_t c, int64_t end, float (&l)[8]) {
    if (c < end) load8<T, false>(row, c, end, l);
#pragma unroll
    for (int i = 0; i < 8; i++) l[i] = c + i < end ? l[i] : NAN;
}
template <typename T>
__device__ __forceinline__ void first_logits(const T *row, int64_t begin, int64_t end, float (&next)[8]) {
    logits8(row, begin + threadIdx.x * 8, end, next);
}
template <typename T, typename F>
__device__ __forceinline__ void each_tile(const T *row, int64_t begin, int64_t end, float (&next)[8], F f) {
    const int64_t own = threadIdx.x * 8;
    for (int64_t c0 = begin; c0 < end; c0 += kTile) {
        float l[8];
#pragma unroll
        for (int i = 0; i < 8; i++) l[i] = next[i];
        if (c0 + kTile < end) logits8(row, c0 + kTile + own, end, next);
        f(l, c0 + own);
    }
}
template <typename T, typename F>
__device__ __forceinline__ void each_tile(const T *row, int64_t begin, int64_t end, F f) {
    float next[8];
    first_logits(row, begin, end, next);
    each_tile(row, begin, end, next, f);
}

// ------------------------------------------------------------------------------------------------ the parts of a row
template <typename T>
__device__ __forceinline__ uint64_t own_best(const T *row, int64_t begin, int64_t end) {  // of a thread's tokens
    uint64_t best = 0;
    each_tile(row, begin, end, [&](const float (&l)[8], int64_t c) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t k = key_of(l[i]);
            if (k) best = max64(best, token_of(k, c + i));
        }
    });
    return best;
}

// top_k without counting the row.  The tokens are in groups; k groups whose largest keys are at least b hold k tokens of at
// least b, so no smaller one is among the k largest.  With twice as many groups as k, a group seldom has many of them: of
// evenly spread tokens 2 k ln 2 = 1.4 k have such a key, which are the list.
constexpr int kMostGroups = 8 * kThreads;
__device__ __forceinline__ bool by_groups(int64_t k, int64_t groups) {
    return k > 0 && k <= kCountOnly && 2 * k <= groups && groups <= kMostGroups;
}

// Such a b from the largest keys of groups (0: none), of which each thread has some, key(i) for i < own; 0 if fewer than k groups have one: by buckets of
// their range, and again of the k-th's bucket while that has more than a quarter of k.
template <typename F>
__device__ __forceinline__ uint32_t bound_of(int own, F key, uint32_t top, int64_t k, Common &sh) {
    uint32_t least = 0;  // its complement
    for (int i = 0; i < own; i++) {
        const uint32_t v = key(i);
        least = max(least, v ? ~v : 0);
    }
    uint64_t low = (uint32_t)~(uint32_t)block_max(least, sh.upart), high = top;
    int64_t wanted = k;
    while (true) {
        int shift = 0;
        while ((high - low) >> shift >= kBuckets) shift++;
        for (int b = threadIdx.x; b < kBuckets; b += kThreads) sh.hist.counts[b] = 0;
        __syncthreads();
        for (int i = 0; i < own; i++) {
            const uint32_t v = key(i);
            if (v && v >= low && v <= high) atomicAdd(&sh.hist.counts[(v - low) >> shift], 1u);
        }
        if (threadIdx.x == 0) sh.found[0] = -1;
        __syncthreads();
        int64_t n[kEach], sum = 0, all;
        const int first = kBuckets - 1 - (int)threadIdx.x * kEach;
#pragma unroll
        for (int i = 0; i < kEach; i++) n[i] = sh.hist.counts[first - i], sum += n[i];
        int64_t upto = block_upto(sum, sh.ipart, all) - sum;
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            if (upto < wanted && upto + n[i] >= wanted) sh.found[0] = first - i, sh.found[1] = upto << 16 | n[i];
            upto += n[i];
        }
        __syncthreads();
        const int64_t bucket = sh.found[0], before = sh.found[1] >> 16, in = sh.found[1] & 0xffff;
        __syncthreads();
        if (bucket < 0) return 0;
        low += (uint64_t)bucket << shift;
        if (shift == 0 || in <= 8 + k / 4) return (uint32_t)low;
        high = min(high, low + (1ull << shift) - 1);
        wanted -= before;
    }
}

// The plan of such a row: its list begins with its first token and ends with the last of at least `bound`.
__device__ __forceinline__ Plan plan_by_groups(const Row &r, uint32_t bound) {
    Plan p;
    p.k = r.top_k, p.before = 0, p.above = p.all = 0.0;
    p.lo = 0, p.hi = row_level().bucket(r.x(bound));
    p.cut_k = true, p.cut_p = r.top_p < 1.0, p.settled = false, p.bound = bound;
    p.top = r.top;
    p.keys = {bound, key_of(r.top) + 1};
    return p;
}

__device__ __forceinline__ void clear(Hist &h) {
    for (int b = threadIdx.x; b < kBuckets; b += kThreads) h.masses[b] = 0, h.counts[b] = 0;
    __syncthreads();
}

template <typename T>
__device__ __forceinline__ void count_buckets(const T *row, int64_t begin, int64_t end, float (&next)[8], const Row &r,
                                              int shift, Hist &h) {
    clear(h);
    const double top = (double)r.top, scale = r.inverse * kPerNat;
    const double magic = magic_of(shift);
    each_tile(row, begin, end, next, [&](const float (&l)[8], int64_t) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            // as r.x and Level::bucket, which are exact in the factor of 16; infinity less itself is 0 here too
            const double y = fmax((top - (double)l[i]) * scale, 0.0);
            const int b = (int)fmin(y, (double)(kBuckets - 1));
            const uint64_t m = (uint64_t)__double_as_longlong(exp_sixteenth(y - (double)b) + magic) & ((1ull << 52) - 1);
            if (!(l[i] > -INFINITY)) continue;
            atomicAdd(&h.counts[b], 1u);
            if (r.masses) atomicAdd((unsigned long long *)&h.masses[b], (unsigned long long)m);
        }
    });
    __syncthreads();
    if (threadIdx.x == 0) h.masses[kBuckets - 1] = 0;
    __syncthreads();
}

// The plan by the buckets in sh.hist.  The row's own has no `outer` one; the one of a list takes from its row's what is known,
// with the tokens and the mass before the list.  masses: whether sh.hist has them.
__device__ __forceinline__ Plan plan_of(const Row &r, const Level &level, bool masses, const Plan *outer, int shift,
                                        Common &sh) {
    Plan p;
    int64_t n[kEach], cells = 0;
    double m[kEach], sum = 0.0;
#pragma unroll
    for (int i = 0; i < kEach; i++) {
        const int b = threadIdx.x * kEach + i;
        n[i] = sh.hist.counts[b];
        m[i] = masses ? ldexp((double)sh.hist.masses[b] * exp(-level.from(b)), -shift) : 0.0;
        cells += n[i], sum += m[i];
    }
    const int64_t base = outer ? outer->before : 0;
    const double under = outer ? outer->above : 0.0;
    int64_t valid;
    const int64_t n0 = base + block_upto(cells, sh.ipart, valid) - cells;
    double listed = 0.0;
    const double m0 = masses ? under + block_upto(sum, sh.part, listed) - sum : 0.0;
    valid += base;
    p.settled = false, p.bound = 0;
    p.top = r.top;
    p.all = outer && r.masses ? outer->all : under + listed;
    p.k = outer ? outer->k : r.top_k > 0 && r.top_k < valid ? r.top_k : valid;
    p.cut_k = outer ? outer->cut_k : p.k < valid;
    p.cut_p = outer ? outer->cut_p : r.top_p < 1.0;
    // the bucket of the k-th token, and the mass before and in it
    if (threadIdx.x == 0) sh.found[0] = kBuckets - 1;
    __syncthreads();
    int64_t c = n0;
    double q = m0;
#pragma unroll
    for (int i = 0; i < kEach; i++) {
        if (c < p.k && c + n[i] >= p.k) sh.found[0] = threadIdx.x * kEach + i, sh.value[0] = q, sh.value[1] = m[i];
        c += n[i], q += m[i];
    }
    __syncthreads();
    const int bucket_k = (int)sh.found[0];
    const double before_k = sh.value[0], in_k = sh.value[1];
    p.lo = kBuckets, p.hi = -1;
    if (!masses) {
        p.lo = 0, p.hi = bucket_k;
    } else {
        if (p.cut_k) p.lo = p.hi = bucket_k;
        if (p.cut_p) {
            // Buckets that may hold the end of the share, whatever part of its bucket the k-th token takes.  Sums by buckets
            // and by tokens differ by less than the slack.
            const double least = r.top_p * (p.cut_k ? before_k : p.all), slack = 1e-12 * (under + listed),
                         most = r.top_p * (p.cut_k ? before_k + in_k : p.all);
            uint64_t first = 0, last = 0;
            q = m0;
#pragma unroll
            for (int i = 0; i < kEach; i++) {
                const int b = threadIdx.x * kEach + i;
                if (n[i] && q - slack < most && q + m[i] + slack >= least)
                    first = max64(first, kBuckets - b), last = max64(last, b + 1);
                q += m[i];
            }
            first = block_max(first, sh.upart);
            if (first) {
                p.lo = min(p.lo, kBuckets - (int)first);
                if (!p.cut_k) p.hi = (int)block_max(last, sh.upart) - 1;
            }
        }
        // where min_p cuts before
        if (r.most_x < (double)INFINITY) {
            const int bucket_m = level.bucket(r.most_x);
            if (bucket_m < p.lo) p.lo = p.hi = bucket_m, p.cut_k = p.cut_p = false;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.found[0] = valid, sh.value[0] = under + listed;  // where all buckets are kept whole
    __syncthreads();
    c = n0, q = m0;
#pragma unroll
    for (int i = 0; i < kEach; i++) {
        if ((int)threadIdx.x * kEach + i == p.lo) sh.found[0] = c, sh.value[0] = q;
        c += n[i], q += m[i];
    }
    __syncthreads();
    p.before = sh.found[0], p.above = sh.value[0];
    __syncthreads();
    return p;
}

// The least key in bucket b or before it, by a wave: a lane tries a 64th of the range each time.
__device__ __forceinline__ uint32_t least_key(const Row &r, int b) {
    const int lane = threadIdx.x % 64;
    const Level level = row_level();
    uint64_t low = key_of(-3.402823466e38f), high = (uint64_t)key_of(r.top) + 1;  // the answer is from low on and before high
    while (high - low > 1) {
        const uint64_t step = (high - low + 63) / 64, at = low + lane * step;
        // keys ascend and buckets descend: lanes from the first that is in bucket b or before
        const bool in = at >= high - 1 || level.bucket(r.x((uint32_t)at)) <= b;
        const int first = __ffsll((unsigned long long)__ballot(in)) - 1;  // -1: not even the last lane's
        if (first == 0) return (uint32_t)low;
        const uint64_t from = low + (uint64_t)(first < 0 ? 63 : first - 1) * step + 1;
        high = first < 0 ? high : min(high, low + (uint64_t)first * step + 1);
        low = from;
    }
    return (uint32_t)low;
}

__device__ __forceinline__ void find_keys(const Row &r, Plan &p, Common &sh) {
    p.keys = {0, 0};
    if (p.hi < p.lo) return;
    const int wave = threadIdx.x / 64;
    if (wave < 2) {
        const uint32_t key = wave == 1 ? least_key(r, p.hi) : p.lo > 0 ? least_key(r, p.lo - 1) : key_of(r.top) + 1;
        if (threadIdx.x % 64 == 0) sh.found[wave] = key;
    }
    __syncthreads();
    p.keys = {(uint32_t)sh.found[1], (uint32_t)sh.found[0]};
    __syncthreads();
}

// put(place, token) for the tokens of the list's buckets in [begin, end), in order of the indices; returns how many there are.
template <typename T, typename F>
__device__ __forceinline__ uint32_t collect(const T *row, int64_t begin, int64_t end, float (&next)[8], const Keys &keys,
                                            uint64_t *part, F put) {
    uint32_t placed = 0;
    each_tile(row, begin, end, next, [&](const float (&l)[8], int64_t c) {
        uint32_t mask = 0;
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (key_of(l[i]) - keys.first < keys.end - keys.first) mask |= 1u << i;
        uint64_t all;
        const int mine = __popc(mask);
        uint32_t at = placed + (uint32_t)block_upto((uint64_t)mine, part, all) - mine;
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (mask >> i & 1) put(at++, token_of(key_of(l[i]), c + i));
        placed += (uint32_t)all;
    });
    return placed;
}
template <typename T, typename F>
__device__ __forceinline__ uint32_t collect(const T *row, int64_t begin, int64_t end, const Plan &p, uint64_t *part, F put) {
    float next[8];
    first_logits(row, begin, end, next);
    return collect(row, begin, end, next, p.keys, part, put);
}

// What is kept of a row (the tokens up to `last` in their order, as far as min_p keeps them), and what is drawn of it.
struct Kept {
    uint64_t last;
    double most_x;
    int64_t count;
    double total, drawn;
    __device__ __forceinline__ bool holds(uint64_t token, double x) const { return token >= last && x <= most_x; }
};

__device__ __forceinline__ void answer(const SampleArgs &a, int64_t at, int64_t id, double prob, int64_t kept) {
    a.ids[at] = (int32_t)id;
    a.prob[at] = (float)prob;
    a.kept[at] = (int32_t)kept;
}

// A row without a token to take, or whose first token is taken: true if that is all.
__device__ __forceinline__ bool settled(const SampleArgs &a, int64_t at, uint64_t best, bool writes) {
    const bool none = best == 0;
    if (!none && !is_greedy(a, at)) return false;
    if (writes && threadIdx.x == 0) answer(a, at, none ? -1 : index_of(best), none ? 0.0 : 1.0, none ? 0 : 1);
    return true;
}

// ------------------------------------------------------------------------------------------------ the list
// Up to a token for each thread: each finds its rank by counting those before it, and everything goes by ranks from there.
// Returns true if the row is answered, which it is where nothing is kept whole before the list.
__device__ __forceinline__ bool by_rank(const SampleArgs &a, int64_t at, const Row &r, const Plan &p, const uint64_t *tokens,
                                        int n, Shared &sh, Kept &kept) {
    const int i = threadIdx.x;
    const bool mine = i < n;
    const uint64_t token = mine ? tokens[i] : 0;
    int rank = 0;
    if ((i & ~63) < n)
#pragma unroll 8
        for (int j = 0; j < n; j++) rank += tokens[j] > token;
    double m = 0.0;
    bool stays = false;
    if (mine) {
        const double x = r.x((uint32_t)(token >> 32));
        m = mass(x, sh.table);
        stays = x <= r.most_x;
        sh.sorted.token[rank] = token, sh.sorted.mass[rank] = m;
    }
    int64_t left = block_sum((int64_t)stays, sh.ipart);  // what min_p leaves; its barriers make the sorted list visible too
    const int64_t left_k = p.cut_k ? p.k - p.before : n;
    left = min(left, left_k);
    if (p.cut_p) {
        double all;
        const double v = mine && i < left_k ? sh.sorted.mass[i] : 0.0, upto = block_upto(v, sh.part, all);
        const double share = !p.cut_k && p.all > 0.0 ? p.all : p.above + all, target = r.top_p * share - p.above;
        // the first that reaches the share, if any does
        const uint64_t reach = block_max(mine && upto >= target ? (uint64_t)(kThreads - i) : 0, sh.upart);
        if (reach) left = min(left, (int64_t)kThreads - (int64_t)reach + 1);
    }
    kept.count = p.before + left;
    if (!mine || rank >= left) m = 0.0;
    double listed;
    const double upto = block_upto(m, sh.part, listed);
    kept.total = p.above + listed;
    kept.drawn = r.u * kept.total;
    kept.last = left > 0 ? sh.sorted.token[left - 1] : sh.sorted.token[0] + 1;
    if (p.before > 0) return false;
    if (i == elect(m > 0.0 && upto > kept.drawn, m > 0.0, sh)) answer(a, at, index_of(token), m / kept.total, kept.count);
    return true;
}

// A longer list in LDS: its tokens are counted again in buckets of a 1024th of its range, and those of the few buckets that
// remain go by rank.  Returns 1 if the row is answered, 0 if not, and -1 if too many tokens remain (equal logits, mostly).
__device__ __forceinline__ int by_zoom(const SampleArgs &a, int64_t at, const Row &r, const Plan &p, int n, int shift,
                                       Shared &sh, Kept &kept) {
    constexpr int kOwn = kList / kThreads;
    const Level level = list_level(p.lo, p.hi);
    clear(sh.hist);
    int b[kOwn];
#pragma unroll
    for (int j = 0; j < kOwn; j++) {
        const int i = threadIdx.x * kOwn + j;
        b[j] = kBuckets;
        if (i >= n) continue;
        const double x = r.x((uint32_t)(sh.list[i] >> 32));
        b[j] = level.bucket(x);
        atomicAdd(&sh.hist.counts[b[j]], 1u);
        atomicAdd((unsigned long long *)&sh.hist.masses[b[j]], (unsigned long long)whole_mass(x, level.from(b[j]), shift));
    }
    __syncthreads();
    const Plan z = plan_of(r, level, true, &p, shift, sh);
    uint64_t mine = 0, left;
#pragma unroll
    for (int j = 0; j < kOwn; j++) mine += b[j] >= z.lo && b[j] <= z.hi;
    uint32_t place = (uint32_t)(block_upto(mine, sh.upart, left) - mine);
    if (left > kRanked) return -1;
    uint64_t in = 0, out = 0;  // of the last token before those buckets, the complement, and the first one after
#pragma unroll
    for (int j = 0; j < kOwn; j++) {
        if (b[j] == kBuckets) continue;
        const uint64_t token = sh.list[threadIdx.x * kOwn + j];
        if (b[j] < z.lo)
            in = max64(in, ~token);
        else if (b[j] > z.hi)
            out = max64(out, token);
        else
            sh.few[place++] = token;
    }
    if (left == 0) {
        in = block_max(in, sh.upart), out = block_max(out, sh.upart);
        kept.count = z.before, kept.total = z.above, kept.drawn = r.u * z.above;
        kept.last = in ? ~in : out + 1;
        return 0;
    }
    __syncthreads();
    return by_rank(a, at, r, z, sh.few, (int)left, sh, kept) ? 1 : 0;
}

// f(token) for every token of the list, a thread's own ones in the same order each time.  n: -1 where it is not in LDS.
template <typename T, typename F>
__device__ __forceinline__ void each_listed(const T *row, int64_t vocab, const Plan &p, int n, const Shared &sh, F f) {
    if (n >= 0) {
        for (int i = threadIdx.x; i < n; i += kThreads) f(sh.list[i]);
        return;
    }
    each_tile(row, 0, vocab, [&](const float (&l)[8], int64_t c) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const uint32_t k = key_of(l[i]);
            if (k - p.keys.first < p.keys.end - p.keys.first) f(token_of(k, c + i));
        }
    });
}

// The first token of the list at which the number of those from `least` on (MASS: the sum of their masses, in units of the
// list's first bucket) reaches `target`: by eight bits of the tokens after the other.
template <bool MASS, typename E>
__device__ __forceinline__ uint64_t select(const Row &r, const Plan &p, uint64_t target, uint64_t least, int shift, Shared &sh,
                                           E each) {
    uint64_t prefix = 0;
    const double from = (double)p.lo / kPerNat;
    for (int low = 56; low >= 0; low -= 8) {
        __syncthreads();
        if (threadIdx.x < kBins) sh.bins.counts[threadIdx.x] = 0, sh.bins.masses[threadIdx.x] = 0;
        __syncthreads();
        each([&](uint64_t token) {
            if (token < least || (low < 56 && token >> (low + 8) != prefix)) return;
            const int b = (int)(token >> low & (kBins - 1));
            atomicAdd(&sh.bins.counts[b], 1u);
            if (MASS) {
                const double x = r.x((uint32_t)(token >> 32));
                if (weighs(x))
                    atomicAdd((unsigned long long *)&sh.bins.masses[b],
                              (unsigned long long)rint(ldexp(exp(from - x), shift)));
            }
        });
        __syncthreads();
        const int b = kBins - 1 - (int)threadIdx.x;  // the largest first
        const bool some = b >= 0 && sh.bins.counts[max(b, 0)] > 0;
        const uint64_t v = !some ? 0 : MASS ? sh.bins.masses[b] : (uint64_t)sh.bins.counts[b];
        uint64_t all;
        const uint64_t upto = block_upto(v, sh.upart, all);
        const int owner = max(elect(some && upto >= target, some, sh), 0);  // the last bin, should the sum not reach it
        if ((int)threadIdx.x == owner) sh.found[0] = (int64_t)(upto - v);
        __syncthreads();
        prefix = prefix << 8 | (uint64_t)(kBins - 1 - min(owner, kBins - 1));
        target -= min(target, (uint64_t)sh.found[0]);
    }
    __syncthreads();
    return prefix;
}

// Any other list, eight passes over it for each cut; where LDS does not hold it (more than kList tokens, or more than an eighth of a
// chunk), over the row, by one workgroup: a top-p that ends in a bucket of thousands of tokens costs a row of 131072 (normal logits of deviation 2
// at temperature 4) 0.5 ms and one of 262144 (at 1.5) 0.8, where 46 us are usual; top_k and top_p both 0.8 and 1.5.
template <typename E>
__device__ __forceinline__ void by_select(const Row &r, const Plan &p, int shift, Shared &sh, Kept &kept, E each) {
    if (p.cut_k) kept.last = select<false>(r, p, (uint64_t)(p.k - p.before), 0, shift, sh, each);
    if (p.cut_p) {
        double share = p.all;
        if (!r.masses || p.cut_k) {
            double sum = 0.0;
            each([&](uint64_t token) {
                if (token >= kept.last) sum += mass(r.x((uint32_t)(token >> 32)), sh.table);
            });
            share = p.above + block_sum(sum, sh.part);
        }
        const double units = ceil(ldexp((r.top_p * share - p.above) * exp((double)p.lo / kPerNat), shift));
        kept.last = select<true>(r, p, units >= 1.0 ? (uint64_t)units : 1, kept.last, shift, sh, each);
    }
    double sum = 0.0;
    int64_t count = 0;
    each([&](uint64_t token) {
        const double x = r.x((uint32_t)(token >> 32));
        if (kept.holds(token, x)) sum += mass(x, sh.table), count++;
    });
    kept.total = p.above + block_sum(sum, sh.part);
    kept.count = p.before + block_sum(count, sh.ipart);
    kept.drawn = r.u * kept.total;
}

// What is kept of the row, from its list of n tokens (which lies in LDS where it fits).  True if the row is answered.
template <typename T>
__device__ __forceinline__ bool keep(const SampleArgs &a, int64_t at, const T *row, const Row &r, const Plan &p, int64_t n,
                                     bool fits, int shift, Shared &sh, Kept &kept) {
    kept = {0, r.most_x, p.before, p.above, r.u * p.above};
    if (n == 0) return false;
    if (fits && n <= kRanked) return by_rank(a, at, r, p, sh.list, (int)n, sh, kept);
    const int done = fits ? by_zoom(a, at, r, p, (int)n, shift, sh, kept) : -1;
    if (done < 0)
        by_select(r, p, shift, sh, kept, [&](auto f) { each_listed(row, a.vocab, p, fits ? (int)n : -1, sh, f); });
    return done > 0;
}

// The masses of the kept ones of eight tokens, and their sum.
__device__ __forceinline__ double kept_masses(const float (&l)[8], int64_t c, const Row &r, const Kept &kept,
                                              const Shared &sh, double (&m)[8]) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        m[i] = 0.0;
        const uint32_t k = key_of(l[i]);
        if (!k) continue;
        const double x = r.x(k);
        if (kept.holds(token_of(k, c + i), x)) m[i] = mass(x, sh.table);
        sum += m[i];
    }
    return sum;
}

// The token within [begin, end), whose kept tokens come after a mass of `before`: each thread takes a run of them, then all
// of them the run in which it lies, until a run is eight tokens.
template <typename T>
__device__ __forceinline__ void draw_in(const SampleArgs &a, int64_t at, const T *row, const Row &r, const Kept &kept,
                                        int64_t begin, int64_t end, double before, Shared &sh) {
    while (true) {
        const int64_t each = (end - begin + kTile - 1) / kTile * 8;
        const int64_t from = min(begin + threadIdx.x * each, end), to = min(from + each, end);
        double m[8], sum = 0.0, all;
        float next[8];
        logits8(row, from, to, next);
        for (int64_t c = from; c < to; c += 8) {
            float l[8];
#pragma unroll
            for (int i = 0; i < 8; i++) l[i] = next[i];
            if (c + 8 < to) logits8(row, c + 8, to, next);
            sum += kept_masses(l, c, r, kept, sh, m);
        }
        const double upto = before + block_upto(sum, sh.part, all);
        const int owner = elect(sum > 0.0 && upto > kept.drawn, sum > 0.0, sh);
        if (owner < 0) {
            if (threadIdx.x == 0) answer(a, at, -1, 0.0, kept.count);
            return;
        }
        if (each == 8) {
            if ((int)threadIdx.x != owner) return;
            double q = upto - sum, taken = 0.0;
            int id = 0;
            bool open = true;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                q += m[i];
                if (open && m[i] > 0.0) id = i, taken = m[i], open = !(q > kept.drawn);
            }
            answer(a, at, from + id, taken / kept.total, kept.count);
            return;
        }
        if ((int)threadIdx.x == owner) sh.found[0] = from, sh.found[1] = to, sh.value[0] = upto - sum;
        __syncthreads();
        begin = sh.found[0], end = sh.found[1], before = sh.value[0];
        __syncthreads();
    }
}

__device__ __forceinline__ void fill_table(Shared &sh) {
    for (int b = threadIdx.x; b < kBuckets; b += kThreads) sh.table[b] = exp(-(double)b / kPerNat);
    __syncthreads();
}

// ------------------------------------------------------------------------------------------------ kernels
// A short row by one workgroup, in one launch.
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_short_kernel(SampleArgs a, int shift) {
    __shared__ Shared sh;
    const int64_t at = blockIdx.x;
    const T *row = (const T *)a.logits + at * a.ld;
    Row r = row_of(a, at);
    const uint64_t own = own_best(row, 0, a.vocab), best = block_max(own, sh.upart);
    if (settled(a, at, best, true)) return;
    r.top = logit_of_key((uint32_t)(best >> 32));
    fill_table(sh);
    uint32_t bound = 0;
    if (by_groups(r.top_k, kThreads))
        bound = bound_of(1, [&](int) { return (uint32_t)(own >> 32); }, (uint32_t)(best >> 32), r.top_k, sh);
    Plan p;
    if (bound) {
        p = plan_by_groups(r, bound);
    } else {
        float next[8];
        first_logits(row, 0, a.vocab, next);
        count_buckets(row, 0, a.vocab, next, r, shift, sh.hist);
        p = plan_of(r, row_level(), r.masses, nullptr, shift, sh);
        find_keys(r, p, sh);
    }
    uint32_t n = 0;
    if (p.hi >= p.lo)
        n = collect(row, 0, a.vocab, p, sh.upart, [&](uint32_t place, uint64_t token) {
            if (place < kList) sh.list[place] = token;
        });
    __syncthreads();
    Kept kept;
    if (keep(a, at, row, r, p, n, n <= kList, shift, sh, kept)) return;
    draw_in(a, at, row, r, kept, 0, a.vocab, 0.0, sh);
}

// The largest keys of a chunk's groups, in its part of ws.parts, which rows with few tokens to keep do not use otherwise.
// lanes: of a group, 1, 8 or 64, so that a row has a few hundred to a few thousand of them.
__device__ __forceinline__ int group_lanes(int64_t chunks) { return chunks < 8 ? 1 : chunks <= 64 ? 8 : 64; }
__device__ __forceinline__ void put_groups(uint32_t key, int lanes, uint32_t *groups) {
    if (lanes > 1) {
        key = max(key, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)key, 0xb1, 0xf, 0xf, true));   // lanes 1 apart
        key = max(key, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)key, 0x4e, 0xf, 0xf, true));   // 2 apart
        key = max(key, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)key, 0x141, 0xf, 0xf, true));  // the other half of eight
    }
    if (lanes > 8) {
        key = max(key, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)key, 0x140, 0xf, 0xf, true));  // of sixteen
        Two t = across16(key);
        t = across32(max(t.a, t.b));
        key = max(t.a, t.b);
    }
    if (threadIdx.x % lanes == 0) groups[threadIdx.x / lanes] = key;
}
__device__ __forceinline__ uint32_t *groups_of(const SampleSpace &ws, int64_t chunk) {
    return (uint32_t *)(ws.parts + chunk * kBuckets);
}

// Longer rows in four launches, the first three by chunks: the first token and the groups' largest keys; the buckets, and the plan by
// whichever workgroup of the row is through last, or the list by the groups; any other list, and the mass of what is kept whole; the end.
// us, float, 131072 tokens, one row with all filters: 3.8, 8.4, 2.1, 7.9, chains of latencies; 128 rows with filters of their own: 15
// (67 MB, 4.4 TB/s), 29, 11, 30.  The rows without top_k are what the last three wait for: a mass and two LDS atomics for each token, then a
// workgroup a row.  A CU that counts four chunks at once takes 1.4 us for 4096 tokens and fills nothing (VALU issue 37%, LDS 10% over the
// call): half the instructions took a tenth off, four copies of the buckets, which spare equal addresses, nothing, and chunks' counts
// summed by the planning workgroup in place of atomics in memory cost 4.
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_best_kernel(SampleArgs a, SampleSpace ws, int64_t chunks, int64_t chunk) {
    __shared__ uint64_t part[kWaves];
    const int64_t at = blockIdx.x / chunks, c = blockIdx.x % chunks;
    for (int64_t b = c * kThreads + threadIdx.x; b < kBuckets; b += chunks * kThreads)
        ws.counts[at * kBuckets + b] = 0, ws.masses[at * kBuckets + b] = 0;
    if (c == 0 && threadIdx.x == 0) ws.done[at] = 0;
    const uint64_t own = own_best((const T *)a.logits + at * a.ld, c * chunk, min((c + 1) * chunk, a.vocab));
    const int lanes = group_lanes(chunks);
    if (by_groups(a.top_k ? a.top_k[at] : 0, chunks * (kThreads / lanes)))
        put_groups((uint32_t)(own >> 32), lanes, groups_of(ws, blockIdx.x));
    const uint64_t best = block_max(own, part);
    if (threadIdx.x == 0) ws.best[blockIdx.x] = best;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_count_kernel(SampleArgs a, SampleSpace ws, int64_t chunks, int64_t chunk,
                                                               int shift) {
    __shared__ Common sh;
    __shared__ uint32_t groups[kMostGroups];
    const int64_t at = blockIdx.x / chunks, c = blockIdx.x % chunks;
    const int64_t begin = c * chunk, end = min(begin + chunk, a.vocab);
    const T *row = (const T *)a.logits + at * a.ld;
    float next[8];
    first_logits(row, begin, end, next);
    uint64_t best = 0;
    for (int64_t w = threadIdx.x; w < chunks; w += kThreads) best = max64(best, ws.best[at * chunks + w]);
    best = block_max(best, sh.upart);
    if (settled(a, at, best, c == 0)) {
        if (c == 0 && threadIdx.x == 0) ws.plan[at].settled = true;
        return;
    }
    const uint32_t top = (uint32_t)(best >> 32);
    const int64_t top_k = a.top_k ? a.top_k[at] : 0;
    const int each = kThreads / group_lanes(chunks);
    if (by_groups(top_k, chunks * each)) {
        const int own = (int)(chunks * each + kThreads - 1) / kThreads;
#pragma unroll 4
        for (int i = 0; i < own; i++) {
            const int g = i * kThreads + threadIdx.x;
            groups[g] = g < chunks * each ? groups_of(ws, at * chunks + g / each)[g % each] : 0;
        }
        const uint32_t bound =
            bound_of(own, [&](int i) { return groups[i * kThreads + threadIdx.x]; }, top, top_k, sh);
        if (bound) {  // or few groups have a token that can be taken, which every workgroup of the row finds alike
            const uint32_t room = (uint32_t)(chunk / 8);
            uint64_t *const list = ws.list + blockIdx.x * (int64_t)room;
            const uint32_t placed = collect(row, begin, end, next, Keys{bound, top + 1}, sh.upart,
                                            [&](uint32_t place, uint64_t token) {
                                                if (place < room) list[place] = token;
                                            });
            if (threadIdx.x == 0) {
                ws.whole[blockIdx.x] = 0.0, ws.listed[blockIdx.x] = placed;
                if (c == 0) ws.plan[at].settled = false, ws.plan[at].bound = bound, ws.plan[at].top = logit_of_key(top);
            }
            return;
        }
    }
    Row r = row_of(a, at);
    r.top = logit_of_key(top);
    count_buckets(row, begin, end, next, r, shift, sh.hist);
    uint32_t *const counts = ws.counts + at * kBuckets;
    unsigned long long *const masses = (unsigned long long *)ws.masses + at * kBuckets;
    for (int b = threadIdx.x; b < kBuckets; b += kThreads) {
        if (r.masses) ws.parts[blockIdx.x * (int64_t)kBuckets + b] = sh.hist.masses[b];
        if (!sh.hist.counts[b]) continue;
        atomicAdd(counts + b, sh.hist.counts[b]);
        if (r.masses) atomicAdd(masses + b, (unsigned long long)sh.hist.masses[b]);
    }
    stores_arrived();
    __syncthreads();
    if (threadIdx.x == 0) sh.found[0] = atomicAdd(ws.done + at, 1u) == (uint32_t)chunks - 1;
    __syncthreads();
    if (!sh.found[0]) return;
    for (int b = threadIdx.x; b < kBuckets; b += kThreads) {
        sh.hist.counts[b] = get_shared(counts + b);
        if (r.masses) sh.hist.masses[b] = get_shared(masses + b);
    }
    __syncthreads();
    Plan p = plan_of(r, row_level(), r.masses, nullptr, shift, sh);
    find_keys(r, p, sh);
    if (threadIdx.x == 0) ws.plan[at] = p;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_list_kernel(SampleArgs a, SampleSpace ws, int64_t chunks, int64_t chunk,
                                                              int shift) {
    __shared__ uint64_t part[kWaves];
    __shared__ double sums[kWaves];
    const int64_t at = blockIdx.x / chunks, c = blockIdx.x % chunks;
    const Plan p = ws.plan[at];
    if (p.settled || p.bound) return;
    const bool masses = row_of(a, at).masses;
    const uint32_t room = (uint32_t)(chunk / 8);
    uint64_t *const list = ws.list + (at * chunks + c) * room;
    uint32_t placed = 0;
    if (p.hi >= p.lo)
        placed = collect((const T *)a.logits + at * a.ld, c * chunk, min((c + 1) * chunk, a.vocab), p, part,
                         [&](uint32_t place, uint64_t token) {
                             if (place < room) list[place] = token;
                         });
    double sum = 0.0;
    if (masses) {
        for (int b = threadIdx.x; b < min(p.lo, kBuckets); b += kThreads)
            sum += ldexp((double)ws.parts[blockIdx.x * (int64_t)kBuckets + b] * exp(-(double)b / kPerNat), -shift);
        sum = block_sum(sum, sums);
    }
    if (threadIdx.x == 0) ws.whole[blockIdx.x] = sum, ws.listed[blockIdx.x] = placed;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_end_kernel(SampleArgs a, SampleSpace ws, int64_t chunks, int64_t chunk,
                                                             int shift) {
    __shared__ Shared sh;
    const int64_t at = blockIdx.x;
    const T *row = (const T *)a.logits + at * a.ld;
    Plan p = ws.plan[at];
    if (p.settled) return;
    Row r = row_of(a, at);
    r.top = p.top;
    if (p.bound) p = plan_by_groups(r, p.bound);
    const uint32_t room = (uint32_t)(chunk / 8);
    double *const whole = ws.whole + at * chunks;
    // the chunks' lists in LDS, where they fit
    int64_t n = 0;
    bool fits = chunks <= kThreads;
    for (int64_t c0 = 0; c0 < chunks; c0 += kThreads) {
        const uint32_t mine = c0 + threadIdx.x < chunks ? ws.listed[at * chunks + c0 + threadIdx.x] : 0;
        int64_t all;
        const int64_t upto = block_upto((int64_t)mine, sh.ipart, all);
        if (c0 == 0) sh.offset[threadIdx.x + 1] = (uint32_t)upto;
        fits = block_max(mine > room, sh.upart) == 0 && fits;
        n += all;
    }
    fits = fits && n <= kList;
    if (threadIdx.x == 0) sh.offset[0] = 0;
    fill_table(sh);
    if (fits && n > 0) {
        constexpr int kOwn = kList / kThreads;
        uint64_t token[kOwn];
#pragma unroll
        for (int j = 0; j < kOwn; j++) {
            const int i = j * kThreads + threadIdx.x;
            int low = 0, high = (int)chunks;  // the chunk of this place: offset[low] <= i < offset[high]
            while (i < n && high - low > 1) {
                const int mid = (low + high) / 2;
                if (sh.offset[mid] <= (uint32_t)i)
                    low = mid;
                else
                    high = mid;
            }
            token[j] = i < n ? ws.list[(at * chunks + low) * room + (i - sh.offset[low])] : 0;
        }
#pragma unroll
        for (int j = 0; j < kOwn; j++) sh.list[j * kThreads + threadIdx.x] = token[j];
        __syncthreads();
    }
    Kept kept;
    if (keep(a, at, row, r, p, n, fits, shift, sh, kept)) return;
    if (n > 0 && fits) {
        // the list's tokens give way to the mass of what is kept of them up to there, and in `upto` to how many have one
        constexpr int kOwn = kList / kThreads;
        double m[kOwn], sum = 0.0, all;
        int64_t weighty = 0, total;
#pragma unroll
        for (int j = 0; j < kOwn; j++) {
            const int i = threadIdx.x * kOwn + j;
            m[j] = 0.0;
            if (i >= n) continue;
            const double x = r.x((uint32_t)(sh.list[i] >> 32));
            if (kept.holds(sh.list[i], x)) m[j] = mass(x, sh.table);
            sum += m[j], weighty += m[j] > 0.0;
        }
        double q = block_upto(sum, sh.part, all) - sum;  // its barriers come between reading and writing
        int64_t n0 = block_upto(weighty, sh.ipart, total) - weighty;
#pragma unroll
        for (int j = 0; j < kOwn; j++) {
            q += m[j], n0 += m[j] > 0.0;
            sh.list[threadIdx.x * kOwn + j] = (uint64_t)__double_as_longlong(q);
            sh.upto[threadIdx.x * kOwn + j] = (uint16_t)n0;
        }
        __syncthreads();
    } else if (n > 0) {
        for (int64_t c = 0; c < chunks; c++) {
            const int64_t end = min((c + 1) * chunk, a.vocab);
            double sum = 0.0;
            double m[8];
            each_tile(row, c * chunk, end,
                      [&](const float (&l)[8], int64_t t) { sum += kept_masses(l, t, r, kept, sh, m); });
            sum = block_sum(sum, sh.part);
            if (threadIdx.x == 0) whole[c] = sum;
        }
        __syncthreads();
    }
    // the chunk whose tokens pass the drawn share, or the last that has any mass
    int64_t chosen = 0;
    double before = 0.0, start = 0.0;
    for (int64_t c0 = 0; c0 < chunks; c0 += kThreads) {
        const int64_t c = c0 + threadIdx.x;
        double m = c < chunks ? whole[c] : 0.0;
        if (n > 0 && fits && c < chunks) {
            // a difference of sums that has a rounding of its own: it is not 0 where nothing is kept
            const uint32_t from = sh.offset[c], to = sh.offset[c + 1];
            if (to > from && sh.upto[to - 1] > (from ? sh.upto[from - 1] : 0))
                m += __longlong_as_double((long long)sh.list[to - 1]) -
                     (from ? __longlong_as_double((long long)sh.list[from - 1]) : 0.0);
        }
        double all;
        const double upto = before + block_upto(m, sh.part, all);
        const bool hit = m > 0.0 && upto > kept.drawn;
        const int owner = elect(hit, m > 0.0, sh);
        if (owner >= 0) {
            if ((int)threadIdx.x == owner) sh.value[0] = upto - m, sh.found[0] = hit;
            chosen = c0 + owner;
            __syncthreads();
            start = sh.value[0];
            if (sh.found[0]) break;
            __syncthreads();
        }
        before += all;
    }
    __syncthreads();
    draw_in(a, at, row, r, kept, chosen * chunk, min((chosen + 1) * chunk, a.vocab), start, sh);
}

// Rows that one workgroup each takes in one launch.  us (this | the four launches), temperature alone, top-p, all filters, float:
//   1 row:      8000 tokens 16, 23, 12 | 25, 33, 23;   16000 24, 33, 15 | 24, 34, 24;   32000 37, 52, 22 | 24, 36, 21
//   128 rows:   32000 39, 53, 22 | 41, 57, 30;   64000 70, 99, 41 | 52, 75, 36;   131072 136, 185, 73 | 71, 100, 50
//   256 rows:   32000 43, 62, 27 | 52, 75, 43;   64000 76, 103, 42 | 70, 97, 51
//   400 rows:   100000 156, 207, 74 | 149, 208, 91
//   512 rows:   64000 108, 143, 56 | 116, 157, 73;   131072 204, 264, 97 | 190, 257, 117
//   600 rows:   131072 305, 406, 163 | 346, 450, 157;   800 rows: 403, 518, 190 | 456, 603, 233
// Which settings a row has is data of the GPU, so the rule goes by the sizes: next to it, rows of all filters win a fifth, others lose up to 9%.
constexpr int64_t kShort = 4 * kTile, kOfARow = 256;
bool is_short(int64_t rows, int64_t vocab) { return vocab <= kShort || vocab / kOfARow <= rows; }

template <typename T>
hipError_t sample_go(const SampleArgs &a, hipStream_t s) {
    int shift = 44;  // a bucket's mass, at most 2^shift for each token, fits 63 bits
    while (shift > 30 && a.vocab >> (63 - shift)) shift--;
    constexpr int64_t kStep = 1 << 22;  // workgroups of a launch, which holds fewer than 2^32 threads
    const int64_t chunk = chunk_of(a.rows, a.vocab), chunks = (a.vocab + chunk - 1) / chunk;
    const int64_t step = is_short(a.rows, a.vocab) ? kStep : kStep / chunks;
    for (int64_t r0 = 0; r0 < a.rows; r0 += step) {
        SampleArgs p = a;
        p.rows = a.rows - r0 < step ? a.rows - r0 : step;
        p.logits = (const T *)a.logits + r0 * a.ld;
        p.uniform += r0;
        if (p.temperature) p.temperature += r0;
        if (p.top_k) p.top_k += r0;
        if (p.top_p) p.top_p += r0;
        if (p.min_p) p.min_p += r0;
        p.ids += r0, p.prob += r0, p.kept += r0;
        if (is_short(a.rows, a.vocab)) {
            sample_short_kernel<T><<<(unsigned)p.rows, kThreads, 0, s>>>(p, shift);
        } else {
            SampleSpace ws;
            sample_sizes(a.rows, a.vocab, a.ws, &ws);
            const unsigned grid = (unsigned)(p.rows * chunks);
            sample_best_kernel<T><<<grid, kThreads, 0, s>>>(p, ws, chunks, chunk);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            sample_count_kernel<T><<<grid, kThreads, 0, s>>>(p, ws, chunks, chunk, shift);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            sample_list_kernel<T><<<grid, kThreads, 0, s>>>(p, ws, chunks, chunk, shift);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            sample_end_kernel<T><<<(unsigned)p.rows, kThreads, 0, s>>>(p, ws, chunks, chunk, shift);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t sample_workspace(int64_t rows, int64_t vocab) {
    return rows == 0 || is_short(rows, vocab) ? 0 : sample_sizes(rows, vocab, nullptr, nullptr);
}

size_t sample_workspace_upto(int64_t rows, int64_t vocab) {
    return sample_workspace(vocab <= kShort ? rows : std::min(rows, vocab / kOfARow - 1), vocab);  // the most that are not short
}

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t stream) {
    if (a.rows == 0) return hipSuccess;
    return bf16 ? sample_go<__bf16>(a, stream) : sample_go<float>(a, stream);
}

}  // namespace sdnn
