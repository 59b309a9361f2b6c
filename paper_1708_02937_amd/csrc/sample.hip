// The next token of each row of logits.
//
//   x_i = (max l - l_i) / temperature,  p_i = exp(-x_i)
//   K = the top_k tokens with the largest logits (equal ones by index),  P = the shortest run of K in that order whose mass is
//   top_p of K's or more,  M = the tokens with p_i >= min_p;  all three are beginnings of one order, and so is what is kept
//   token = the first index at which the mass of the kept tokens up to it exceeds u times the mass of all of them
//
// Which token it is goes by sums in 64 bits: 32 do not tell the tokens of a large vocabulary apart.  Nothing is sorted.  A
// row's tokens are counted in buckets of x, a 16th wide, with their mass as whole numbers, so that the order of the additions
// does not matter; the buckets tell where the order ends, within a bucket or a few, and only the tokens of those are looked
// at one by one.  Buckets above them are kept whole.
//
// A bucket's masses are in units of exp(-b / 16) 2^-shift: e^-d for 0 <= d < 1/16 is a polynomial of degree 8 (the next term is
// 4e-17), and the sum of a bucket is as exact as its values.  The last bucket is x >= 63.9: its tokens count, but their mass,
// below 2e-28 of the first token's each, is 0.
#include "blocks8.h"
#include "common.h"
#include "lanes.h"
#include "shared_memory.h"

namespace sdnn {
namespace {

constexpr int kThreads = 512, kWaves = kThreads / 64;
constexpr int kTile = kThreads * 8;   // tokens that a workgroup looks at in turn
constexpr int kBuckets = 1024, kPerNat = 16;
constexpr int kList = 4096;           // tokens of the last buckets that fit LDS; more are looked for in the row each time
constexpr int kSorted = kThreads;     // up to so many are ranked by counting
constexpr int kCountOnly = 1024;      // up to so many tokens kept by top_k, masses are not summed over the row
constexpr int kBins = 2048;           // of one level of a selection by the bits of a logit: 11, 11 and 10 of them

// The order of logits as numbers above 0; 0 for one that cannot be taken (-inf, NaN).
__device__ __forceinline__ uint32_t key_of(float l) {
    if (!(l > -INFINITY)) return 0;
    const uint32_t b = __float_as_uint(l + 0.0f);  // -0 is 0
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of_key(uint32_t k) {
    return __uint_as_float(k ^ ((k >> 31) ? 0x80000000u : 0xffffffffu));
}

struct Row {
    int64_t vocab;
    float top;  // largest logit
    double inverse;  // of the temperature
    double most_x;   // x of min_p
    int shift;

    __device__ __forceinline__ double x(float l) const { return l == top ? 0.0 : ((double)top - (double)l) * inverse; }
    __device__ __forceinline__ static int bucket(double x) { return (int)fmin(x * kPerNat, (double)(kBuckets - 1)); }
};

// e^-d, 0 <= d <= 1/16.
__device__ __forceinline__ double exp_small(double d) {
    double e = 1.0 / 40320.0;
    e = fma(-d, e, 1.0 / 5040.0), e = fma(-d, e, 1.0 / 720.0), e = fma(-d, e, 1.0 / 120.0), e = fma(-d, e, 1.0 / 24.0);
    e = fma(-d, e, 1.0 / 6.0), e = fma(-d, e, 0.5), e = fma(-d, e, 1.0);
    return fma(-d, e, 1.0);
}

// The mass of x in its bucket's unit, a whole number of 2^-shift.
__device__ __forceinline__ uint64_t whole_mass(const Row &r, double x, int b) {
    if (b == kBuckets - 1) return 0;
    const double magic = __hiloint2double((1023 + 52 - r.shift) << 20, 0);  // its last place is 2^-shift
    return (uint64_t)__double_as_longlong(exp_small(x - (double)b / kPerNat) + magic) & ((1ull << 52) - 1);
}

__device__ __forceinline__ double mass(double x) { return x * kPerNat < (double)(kBuckets - 1) ? exp(-x) : 0.0; }

struct SampleSpace {
    uint64_t *best;      // rows x chunks: largest key and the complement of its first index
    uint32_t *done;      // rows: chunks that are through with the last kernel
    uint32_t *counts;    // rows x buckets
    uint64_t *masses;    // rows x buckets
    uint64_t *parts;     // rows x chunks x buckets: the chunk's masses
    double *whole;       // rows x chunks: mass of the chunk's tokens in buckets that are kept whole
    uint32_t *listed;    // rows x chunks: tokens in the buckets that are looked at one by one
    uint32_t *list;      // rows x chunks x chunk / 8 of their indices
};

// Tokens of a chunk: whole tiles, so that a call has about 1024 workgroups.
int64_t tiles_of(int64_t vocab) { return (vocab + kTile - 1) / kTile; }
int64_t chunk_of(int64_t rows, int64_t vocab) {
    const int64_t each = rows < 1024 ? 1024 / rows : 1;
    return (tiles_of(vocab) + each - 1) / each * kTile;
}

struct SampleSizes {
    size_t done, counts, masses, parts, whole, listed, list, bytes;
};

// Of bounds that grow with the rows, so that the space for the most rows holds any call of fewer.
SampleSizes sample_sizes(int64_t rows, int64_t vocab) {
    const int64_t tiles = tiles_of(vocab), chunk = chunk_of(rows, vocab);
    const size_t most = rows < 1024 ? 1024 : rows, chunks = (size_t)(rows < (int64_t)most / tiles ? rows * tiles : most);
    SampleSizes s;
    s.masses = align_up(chunks * 8);
    s.parts = s.masses + align_up(rows * kBuckets * 8);
    s.whole = s.parts + align_up(chunks * kBuckets * 8);
    s.counts = s.whole + align_up(chunks * 8);
    s.listed = s.counts + align_up(rows * kBuckets * 4);
    s.list = s.listed + align_up(chunks * 4);
    s.done = s.list + align_up((size_t)rows * (tiles * kTile + chunk - kTile) / 8 * 4);
    s.bytes = s.done + align_up(rows * 4);
    return s;
}

SampleSpace sample_space(void *ws, int64_t rows, int64_t vocab) {
    const SampleSizes s = sample_sizes(rows, vocab);
    char *p = (char *)ws;
    return {(uint64_t *)p,           (uint32_t *)(p + s.done), (uint32_t *)(p + s.counts), (uint64_t *)(p + s.masses),
            (uint64_t *)(p + s.parts), (double *)(p + s.whole), (uint32_t *)(p + s.listed), (uint32_t *)(p + s.list)};
}

// ------------------------------------------------------------------------------------------------ over a workgroup
__device__ __forceinline__ uint64_t max64(uint64_t a, uint64_t b) { return a > b ? a : b; }

__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t *part) {
    for (int m = 1; m < 64; m <<= 1) v = max64(v, __shfl_xor((unsigned long long)v, m));
    __syncthreads();
    if (threadIdx.x % 64 == 0) part[threadIdx.x / 64] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kWaves; w++) v = max64(v, part[w]);
    return v;
}

template <typename V>
__device__ __forceinline__ V wave_upto(V v) {
    const int lane = threadIdx.x % 64;
    for (int m = 1; m < 64; m <<= 1) {
        const V o = __shfl_up(v, m);
        if (lane >= m) v += o;
    }
    return v;
}

// The sum of the threads' values up to this one's, and of all.
template <typename V>
__device__ __forceinline__ V block_upto(V v, V *part, V &all) {
    const int wave = threadIdx.x / 64;
    V upto = wave_upto(v);
    __syncthreads();
    if (threadIdx.x % 64 == 63) part[wave] = upto;
    __syncthreads();
    all = V(0);
    V before = V(0);
    for (int w = 0; w < kWaves; w++) {
        if (w == wave) before = all;
        all += part[w];
    }
    return before + upto;
}

template <typename V>
__device__ __forceinline__ V block_sum(V v, V *part) {
    V all;
    block_upto(v, part, all);
    return all;
}

// Eight logits of a row from token c on, as keys.
template <typename T>
__device__ __forceinline__ void keys8(const T *row, int64_t c, int64_t end, uint32_t (&k)[8]) {
    float l[8];
    if (c < end) load8<T, false>(row, c, end, l);
#pragma unroll
    for (int i = 0; i < 8; i++) k[i] = c + i < end ? key_of(l[i]) : 0;
}

// ------------------------------------------------------------------------------------------------ the parts of a row
template <typename T>
__device__ __forceinline__ uint64_t best_of(const T *row, int64_t begin, int64_t end, uint64_t *part) {
    uint64_t best = 0;
    for (int64_t c = begin + threadIdx.x * 8; c < end; c += kTile) {
        uint32_t k[8];
        keys8(row, c, end, k);
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (k[i]) best = max64(best, (uint64_t)k[i] << 32 | (uint32_t)~(uint32_t)(c + i));
    }
    return block_max(best, part);
}

struct Hist {
    uint64_t masses[kBuckets];
    uint32_t counts[kBuckets];
};

__device__ __forceinline__ void clear(Hist &h) {
    for (int b = threadIdx.x; b < kBuckets; b += kThreads) h.masses[b] = 0, h.counts[b] = 0;
}

template <typename T>
__device__ __forceinline__ void count_buckets(const T *row, int64_t begin, int64_t end, const Row &r, bool masses, Hist &h) {
    for (int64_t c = begin + threadIdx.x * 8; c < end; c += kTile) {
        uint32_t k[8];
        keys8(row, c, end, k);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (!k[i]) continue;
            const double x = r.x(logit_of_key(k[i]));
            const int b = Row::bucket(x);
            atomicAdd(&h.counts[b], 1u);
            if (masses) atomicAdd((unsigned long long *)&h.masses[b], (unsigned long long)whole_mass(r, x, b));
        }
    }
}

// Settings of a row.
struct Settings {
    double temperature, top_p, min_p, u;
    int64_t top_k;
    bool greedy, masses;
};

__device__ __forceinline__ Settings settings_of(const SampleArgs &a, int64_t row) {
    Settings s;
    s.temperature = a.temperature ? (double)a.temperature[row] : 1.0;
    s.top_k = a.top_k ? a.top_k[row] : 0;
    s.top_p = a.top_p ? (double)a.top_p[row] : 1.0;
    s.min_p = a.min_p ? (double)a.min_p[row] : 0.0;
    if (s.top_p < 0.0) s.top_p = 0.0;
    s.u = a.uniform[row];
    s.greedy = !(s.temperature > 0.0);
    if (s.temperature == (double)INFINITY) s.temperature = 1e300;  // every token alike
    s.masses = !(s.top_k > 0 && s.top_k <= kCountOnly);
    return s;
}

__device__ __forceinline__ Row row_of(const SampleArgs &a, const Settings &s, float top, int shift) {
    Row r;
    r.vocab = a.vocab, r.top = top, r.inverse = 1.0 / s.temperature, r.shift = shift;
    r.most_x = s.min_p > 0.0 ? -log(fmin(s.min_p, 1.0)) : (double)INFINITY;
    return r;
}

// What the buckets tell of a row.
constexpr int kEach = kBuckets / kThreads;  // buckets of a thread
struct Plan {
    int64_t k;          // tokens that top_k leaves
    bool cut_k, cut_p;  // whether there is anything to cut
    int lo, hi;         // buckets that are looked at token by token; those before are kept whole
    int64_t before;     // tokens of the buckets before lo, and their mass
    double above;
    double all;          // the row's mass (0 where masses are not summed)
    double unit[kEach];  // of the thread's buckets' masses
};

struct Shared {
    union {
        Hist hist;
        struct {
            uint64_t masses[kBins];
            uint32_t counts[kBins];
        } bins;
        struct {
            uint32_t key[kSorted], index[kSorted];
            double mass[kSorted];
            double upto[kSorted + 1];
        } sorted;
    };
    uint32_t key[kList], index[kList];  // the list, in order of the indices
    double part[kWaves];
    uint64_t upart[kWaves];
    int64_t ipart[kWaves];
    int64_t found[4];
    double value[2];
    uint32_t offset[kThreads + 1];  // of the chunks' parts of the list
    uint32_t last;
};

__device__ __forceinline__ Plan plan_of(const Settings &s, const Row &r, Shared &sh) {
    Plan p;
    int64_t n[kEach], cells = 0;
    double m[kEach], sum = 0.0;
#pragma unroll
    for (int i = 0; i < kEach; i++) {
        const int b = threadIdx.x * kEach + i;
        n[i] = sh.hist.counts[b];
        p.unit[i] = s.masses ? ldexp(exp(-(double)b / kPerNat), -r.shift) : 0.0;
        m[i] = s.masses ? (double)sh.hist.masses[b] * p.unit[i] : 0.0;
        cells += n[i], sum += m[i];
    }
    int64_t valid;
    const int64_t n0 = block_upto(cells, sh.ipart, valid) - cells;
    p.all = 0.0;
    const double m0 = s.masses ? block_upto(sum, sh.part, p.all) - sum : 0.0;
    p.k = s.top_k > 0 && s.top_k < valid ? s.top_k : valid;
    p.cut_k = p.k < valid;
    p.cut_p = s.top_p < 1.0;
    // the bucket of the k-th token, and the mass before and in it
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
    if (!s.masses) {
        p.lo = 0, p.hi = bucket_k;
    } else {
        if (p.cut_k) p.lo = p.hi = bucket_k;
        if (p.cut_p) {
            // Buckets that may hold the end of the share, whatever part of its bucket the k-th token takes.  Sums by buckets
            // and by tokens differ by less than the slack.
            const double slack = 1e-12 * p.all, least = s.top_p * (p.cut_k ? before_k : p.all),
                         most = s.top_p * (p.cut_k ? before_k + in_k : p.all);
            uint64_t first = 0, last = 0;
            q = m0;
#pragma unroll
            for (int i = 0; i < kEach; i++) {
                const int b = threadIdx.x * kEach + i;
                if (n[i] && q - slack < most && q + m[i] + slack >= least)
                    first = max64(first, kBuckets - b), last = max64(last, b + 1);
                q += m[i];
            }
            first = block_max(first << 32 | last, sh.upart);  // the first bucket's `last` does not matter with one alone
            if (first >> 32) {
                p.lo = min(p.lo, kBuckets - (int)(first >> 32));
                if (!p.cut_k) p.hi = (int)block_max(last, sh.upart) - 1;
            }
        }
        // where min_p cuts before
        if (r.most_x < (double)INFINITY) {
            const int bucket_m = Row::bucket(r.most_x);
            if (bucket_m < p.lo) p.lo = p.hi = bucket_m, p.cut_k = p.cut_p = false;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) sh.found[0] = valid, sh.value[0] = p.all;  // of a row whose buckets are all kept whole
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

// The indices of the tokens in buckets lo to hi among [begin, end), in order, to put(place, index, key); returns how many
// places there are then.
template <typename T, typename F>
__device__ __forceinline__ uint32_t collect(const T *row, int64_t begin, int64_t end, const Row &r, const Plan &p, Shared &sh,
                                            F put) {
    uint32_t placed = 0;
    for (int64_t c0 = begin; c0 < end; c0 += kTile) {
        const int64_t c = c0 + threadIdx.x * 8;
        uint32_t k[8], mask = 0;
        keys8(row, c, end, k);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const int b = k[i] ? Row::bucket(r.x(logit_of_key(k[i]))) : kBuckets;
            if (b >= p.lo && b <= p.hi) mask |= 1u << i;
        }
        uint64_t all;
        const int mine = __popc(mask);
        uint32_t at = placed + (uint32_t)block_upto((uint64_t)mine, sh.upart, all) - mine;
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (mask >> i & 1) put(at++, (uint32_t)(c + i), k[i]);
        placed += (uint32_t)all;
    }
    return placed;
}

// The tokens of the last buckets: in LDS, or, where they are too many, looked for in the row.
template <typename T>
struct Listed {
    const T *row;
    const Row &r;
    const Plan &p;
    Shared &sh;
    int n;  // -1: not in LDS

    // f(key, index) for every one of them, in any order; a thread's own ones in the same order each time
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
        if (n >= 0) {
            for (int i = threadIdx.x; i < n; i += kThreads) f(sh.key[i], sh.index[i]);
            return;
        }
        for (int64_t c = threadIdx.x * 8; c < r.vocab; c += kTile) {
            uint32_t k[8];
            keys8(row, c, r.vocab, k);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                if (!k[i]) continue;
                const int b = Row::bucket(r.x(logit_of_key(k[i])));
                if (b >= p.lo && b <= p.hi) f(k[i], (uint32_t)(c + i));
            }
        }
    }
};

// The index of the rank-th token with that key (from 1 on) in order of the indices.
template <typename T>
__device__ __forceinline__ int64_t nth_equal(const Listed<T> &l, uint32_t key, int64_t rank, Shared &sh) {
    int64_t before = 0;
    if (l.n >= 0) {
        for (int c0 = 0; c0 < l.n; c0 += kThreads) {
            const int i = c0 + threadIdx.x;
            const bool equal = i < l.n && sh.key[i] == key;
            int64_t all;
            const int64_t upto = before + block_upto((int64_t)equal, sh.ipart, all);
            if (equal && upto == rank) sh.found[0] = sh.index[i];
            before += all;
        }
        __syncthreads();
        return sh.found[0];
    }
    const T *row = l.row;
    const int64_t vocab = l.r.vocab;
    for (int64_t c0 = 0; c0 < vocab; c0 += kTile) {
        const int64_t c = c0 + threadIdx.x * 8;
        uint32_t k[8];
        keys8(row, c, vocab, k);
        int mine = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) mine += k[i] == key;
        int64_t all;
        int64_t at = before + block_upto((int64_t)mine, sh.ipart, all) - mine;
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (k[i] == key && ++at == rank) sh.found[0] = c + i;
        before += all;
        __syncthreads();
        if (before >= rank) break;
    }
    return sh.found[0];
}

// Where an order ends: tokens with a larger key are in, those with this one up to the index.
struct End {
    uint32_t key = 0;
    int64_t index = 0;
    __device__ __forceinline__ bool holds(uint32_t k, int64_t i) const { return k > key || (k == key && i <= index); }
};

// The first of the listed tokens that are `in`, largest keys first, at which their number (MASS: the sum of their masses, in
// units of the first bucket's) reaches `target`.
template <bool MASS, typename T, typename F>
__device__ __forceinline__ End select(const Listed<T> &l, uint64_t target, Shared &sh, F in) {
    uint32_t prefix = 0;
    int64_t equal = 0;
    const double from = (double)l.p.lo / kPerNat, scale = ldexp(1.0, l.r.shift);
    auto units = [&](uint32_t key) {
        const double x = l.r.x(logit_of_key(key));
        return x * kPerNat < (double)(kBuckets - 1) ? (uint64_t)rint(exp(from - x) * scale) : 0ull;
    };
    for (int level = 0; level < 3; level++) {
        const int shift = level == 0 ? 21 : level == 1 ? 10 : 0, width = level == 2 ? 10 : 11;
        __syncthreads();
        for (int b = threadIdx.x; b < kBins; b += kThreads) sh.bins.counts[b] = 0, sh.bins.masses[b] = 0;
        __syncthreads();
        l.each([&](uint32_t key, uint32_t index) {
            if (level > 0 && key >> (shift + width) != prefix) return;
            if (!in(key, index)) return;
            const uint32_t b = key >> shift & ((1u << width) - 1);
            atomicAdd(&sh.bins.counts[b], 1u);
            if (MASS) atomicAdd((unsigned long long *)&sh.bins.masses[b], (unsigned long long)units(key));
        });
        __syncthreads();
        constexpr int kEach = kBins / kThreads;
        uint64_t v[kEach], sum = 0;
        uint64_t lowest = 0;
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            const int b = kBins - 1 - (threadIdx.x * kEach + i);
            v[i] = MASS ? sh.bins.masses[b] : (uint64_t)sh.bins.counts[b];
            if (sh.bins.counts[b]) lowest = kBins - b;
            sum += v[i];
        }
        uint64_t all;
        uint64_t before = block_upto(sum, sh.upart, all) - sum;
        lowest = block_max(lowest, sh.upart);  // the order's end, should the sum not reach the target
        if (target > all) target = all;
        if (threadIdx.x == 0) sh.found[0] = kBins - (int64_t)lowest, sh.found[1] = (int64_t)target, sh.found[2] = 0;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            const int b = kBins - 1 - (threadIdx.x * kEach + i);
            if (before < target && before + v[i] >= target) sh.found[0] = b, sh.found[1] = (int64_t)before, sh.found[2] = 1;
            before += v[i];
        }
        __syncthreads();
        const uint32_t b = min((uint32_t)sh.found[0], (uint32_t)kBins - 1);
        prefix = prefix << width | b;
        if (sh.found[2]) target -= (uint64_t)sh.found[1];
        equal = sh.bins.counts[b];
    }
    int64_t rank = (int64_t)target;
    if (MASS) {
        const uint64_t one = units(prefix);
        rank = one ? (int64_t)((target + one - 1) / one) : equal;
    }
    rank = rank < 1 ? 1 : rank;
    End end;
    end.key = prefix;
    end.index = rank >= equal ? l.r.vocab : nth_equal(l, prefix, rank, sh);
    __syncthreads();
    return end;
}

// What is kept of a row, and what is drawn of it.
struct Kept {
    End k, p;
    double most_x;
    int64_t count;
    double total, drawn;
    __device__ __forceinline__ bool holds(uint32_t key, int64_t index, double x) const {
        return k.holds(key, index) && p.holds(key, index) && x <= most_x;
    }
};

__device__ __forceinline__ Kept all_of(const Settings &s, const Row &r, const Plan &p) {
    Kept k;
    k.most_x = r.most_x, k.count = p.before, k.total = p.above, k.drawn = s.u * p.above;
    return k;
}

__device__ __forceinline__ void answer(const SampleArgs &a, int64_t at, int64_t id, double prob, int64_t kept) {
    a.ids[at] = (int32_t)id;
    a.prob[at] = (float)prob;
    a.kept[at] = (int32_t)kept;
}

// The token within [begin, end), whose kept tokens come after a mass of `before`: a thread takes a run of them.
template <typename T>
__device__ __forceinline__ void draw_in(const SampleArgs &a, int64_t at, const T *row, const Row &r, const Kept &kept,
                                        int64_t begin, int64_t end, double before, Shared &sh) {
    const int64_t each = (end - begin + kTile - 1) / kTile * 8;
    const int64_t from = min(begin + threadIdx.x * each, end), to = min(from + each, end);
    double sum = 0.0;
    for (int64_t c = from; c < to; c += 8) {
        uint32_t k[8];
        keys8(row, c, to, k);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            if (!k[i]) continue;
            const double x = r.x(logit_of_key(k[i]));
            if (kept.holds(k[i], c + i, x)) sum += mass(x);
        }
    }
    double all;
    const double upto = before + block_upto(sum, sh.part, all);
    // the thread whose run passes the drawn share, or the last that has any mass
    const uint64_t first = block_max(sum > 0.0 && upto > kept.drawn ? kThreads - threadIdx.x : 0, sh.upart);
    const uint64_t any = block_max(sum > 0.0 ? threadIdx.x + 1 : 0, sh.upart);
    if (!any) {
        if (threadIdx.x == 0) answer(a, at, -1, 0.0, kept.count);
        return;
    }
    if ((int64_t)threadIdx.x != (first ? kThreads - (int64_t)first : (int64_t)any - 1)) return;
    double q = upto - sum, last = 0.0;
    int64_t id = -1;
    for (int64_t c = from; c < to; c++) {
        const uint32_t k = key_of(load_f32(row + c));
        if (!k) continue;
        const double x = r.x(logit_of_key(k));
        const double m = kept.holds(k, c, x) ? mass(x) : 0.0;
        if (!(m > 0.0)) continue;
        id = c, last = m;
        q += m;
        if (q > kept.drawn) break;
    }
    answer(a, at, id, last / kept.total, kept.count);
}

// A list of up to a token for each thread: each finds its rank by counting the larger ones, and everything goes by ranks from
// there.  Leaves in sh.sorted.upto the mass of the kept ones among the list's first so many.  Returns true if the token is drawn
// and answered, which it is where no bucket is kept whole.
__device__ __forceinline__ bool by_rank(const SampleArgs &a, int64_t at, const Settings &s, const Row &r, const Plan &p, int n,
                                        Shared &sh, Kept &kept) {
    const int i = threadIdx.x;
    const bool mine = i < n;
    const uint32_t key = mine ? sh.key[i] : 0;
    int rank = 0;
    if ((i & ~63) < n) {  // equal ones before a token are larger, and equal ones after it are not
        const int w0 = i & ~63, w1 = min(w0 + 64, n);
#pragma unroll 8
        for (int j = 0; j < w0; j++) rank += sh.key[j] >= key;
        for (int j = w0; j < w1; j++) rank += sh.key[j] > key || (sh.key[j] == key && j < i);
#pragma unroll 8
        for (int j = w1; j < n; j++) rank += sh.key[j] > key;
    }
    double m = 0.0;
    bool stays = false;
    if (mine) {
        const double x = r.x(logit_of_key(key));
        m = mass(x);
        stays = x <= r.most_x;
        sh.sorted.key[rank] = key, sh.sorted.index[rank] = sh.index[i], sh.sorted.mass[rank] = m;
    }
    int64_t left = block_sum((int64_t)stays, sh.ipart);  // what min_p leaves; its barriers make the sorted list visible too
    const int64_t left_k = p.cut_k ? p.k - p.before : n;
    left = min(left, left_k);
    if (p.cut_p) {
        double all;
        const double v = mine && i < left_k ? sh.sorted.mass[i] : 0.0, upto = block_upto(v, sh.part, all);
        const double share = s.masses && !p.cut_k ? p.all : p.above + all, target = s.top_p * share - p.above;
        // the first that reaches the share, if any does
        const uint64_t reach = block_max(mine && upto >= target ? (uint64_t)(kThreads - i) : 0, sh.upart);
        if (reach) left = min(left, (int64_t)kThreads - (int64_t)reach + 1);
    }
    kept.count = p.before + left;
    if (!mine || rank >= left) m = 0.0;
    double listed;
    const double upto = block_upto(m, sh.part, listed);
    kept.total = p.above + listed;
    kept.drawn = s.u * kept.total;
    if (p.lo == 0) {
        const uint64_t first = block_max(m > 0.0 && upto > kept.drawn ? (uint64_t)(kThreads - i) : 0, sh.upart);
        const uint64_t any = first ? 1 : block_max(m > 0.0 ? (uint64_t)(i + 1) : 0, sh.upart);
        if (i == (first ? kThreads - (int)first : (int)any - 1)) answer(a, at, sh.index[i], m / kept.total, kept.count);
        return true;
    }
    if (i == 0) sh.sorted.upto[0] = 0.0;
    sh.sorted.upto[i + 1] = upto;
    // the kept tokens of the list are those up to the last one's place in the order
    kept.k.key = sh.sorted.key[left > 0 ? left - 1 : 0];
    kept.k.index = (int64_t)sh.sorted.index[left > 0 ? left - 1 : 0] - (left > 0 ? 0 : 1);
    __syncthreads();
    return false;
}

// Longer lists.
template <typename T>
__device__ __forceinline__ void by_select(const Settings &s, const Row &r, const Plan &p, const Listed<T> &l, Shared &sh,
                                          Kept &kept) {
    if (p.cut_k) kept.k = select<false>(l, (uint64_t)(p.k - p.before), sh, [](uint32_t, uint32_t) { return true; });
    if (p.cut_p) {
        double share = p.all;
        if (!s.masses || p.cut_k) {
            double sum = 0.0;
            l.each([&](uint32_t k, uint32_t i) {
                if (kept.k.holds(k, i)) sum += mass(r.x(logit_of_key(k)));
            });
            share = p.above + block_sum(sum, sh.part);
        }
        const double units = ceil((s.top_p * share - p.above) * exp((double)p.lo / kPerNat) * ldexp(1.0, r.shift));
        kept.p = select<true>(l, units >= 1.0 ? (uint64_t)units : 1ull, sh,
                              [&](uint32_t k, uint32_t i) { return kept.k.holds(k, i); });
    }
    double sum = 0.0;
    int64_t count = 0;
    l.each([&](uint32_t k, uint32_t i) {
        const double x = r.x(logit_of_key(k));
        if (kept.holds(k, i, x)) sum += mass(x), count++;
    });
    kept.total = p.above + block_sum(sum, sh.part);
    kept.count = p.before + block_sum(count, sh.ipart);
    kept.drawn = s.u * kept.total;
}

// A row without a token to take, or whose largest logit is taken: true if that is all.
__device__ __forceinline__ bool settled(const SampleArgs &a, int64_t at, const Settings &s, uint64_t best, bool writes) {
    const bool none = best == 0;
    if (!none && !s.greedy) return false;
    if (writes && threadIdx.x == 0) {
        answer(a, at, none ? -1 : (int32_t)~(uint32_t)best, none ? 0.0 : 1.0, none ? 0 : 1);
    }
    return true;
}

// ------------------------------------------------------------------------------------------------ kernels
// A short row by one workgroup, in one launch.
constexpr int64_t kShort = 8 * kTile;

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_short_kernel(SampleArgs a, int shift) {
    __shared__ Shared sh;
    const int64_t at = blockIdx.x;
    const T *row = (const T *)a.logits + at * a.ld;
    const Settings s = settings_of(a, at);
    const uint64_t best = best_of(row, 0, a.vocab, sh.upart);
    if (settled(a, at, s, best, true)) return;
    const Row r = row_of(a, s, logit_of_key((uint32_t)(best >> 32)), shift);
    clear(sh.hist);
    __syncthreads();
    count_buckets(row, 0, a.vocab, r, s.masses, sh.hist);
    __syncthreads();
    const Plan p = plan_of(s, r, sh);
    uint32_t n = 0;
    if (p.hi >= 0)
        n = collect(row, 0, a.vocab, r, p, sh, [&](uint32_t place, uint32_t index, uint32_t key) {
            if (place < kList) sh.key[place] = key, sh.index[place] = index;
        });
    __syncthreads();
    Kept kept = all_of(s, r, p);
    if (n > 0 && n <= kSorted) {
        if (by_rank(a, at, s, r, p, (int)n, sh, kept)) return;
    } else if (n > 0) {
        by_select(s, r, p, Listed<T>{row, r, p, sh, n <= kList ? (int)n : -1}, sh, kept);
    }
    draw_in(a, at, row, r, kept, 0, a.vocab, 0.0, sh);
}

// Longer ones in three: the largest logit of each chunk; the buckets; the list, and the row's end by whichever workgroup
// of the row is through last.
template <typename T>
__global__ void __launch_bounds__(kThreads) sample_best_kernel(SampleArgs a, SampleSpace ws, int64_t chunks, int64_t chunk) {
    __shared__ uint64_t part[kWaves];
    const int64_t at = blockIdx.x / chunks, c = blockIdx.x % chunks;
    for (int64_t b = c * kThreads + threadIdx.x; b < kBuckets; b += chunks * kThreads)
        ws.counts[at * kBuckets + b] = 0, ws.masses[at * kBuckets + b] = 0;
    if (c == 0 && threadIdx.x == 0) ws.done[at] = 0;
    const uint64_t best = best_of((const T *)a.logits + at * a.ld, c * chunk, min((c + 1) * chunk, a.vocab), part);
    if (threadIdx.x == 0) ws.best[blockIdx.x] = best;
}

__device__ __forceinline__ uint64_t row_best(const SampleSpace &ws, int64_t at, int64_t chunks, uint64_t *part) {
    uint64_t best = 0;
    for (int64_t c = threadIdx.x; c < chunks; c += kThreads) best = max64(best, ws.best[at * chunks + c]);
    return block_max(best, part);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_count_kernel(SampleArgs a, SampleSpace ws, int64_t chunks, int64_t chunk,
                                                               int shift) {
    __shared__ Hist hist;
    __shared__ uint64_t part[kWaves];
    const int64_t at = blockIdx.x / chunks, c = blockIdx.x % chunks;
    const Settings s = settings_of(a, at);
    const uint64_t best = row_best(ws, at, chunks, part);
    if (settled(a, at, s, best, c == 0)) return;
    const Row r = row_of(a, s, logit_of_key((uint32_t)(best >> 32)), shift);
    clear(hist);
    __syncthreads();
    count_buckets((const T *)a.logits + at * a.ld, c * chunk, min((c + 1) * chunk, a.vocab), r, s.masses, hist);
    __syncthreads();
    for (int b = threadIdx.x; b < kBuckets; b += kThreads) {
        if (!hist.counts[b]) continue;
        atomicAdd(&ws.counts[at * kBuckets + b], hist.counts[b]);
        if (s.masses) atomicAdd((unsigned long long *)&ws.masses[at * kBuckets + b], (unsigned long long)hist.masses[b]);
    }
    if (s.masses)
        for (int b = threadIdx.x; b < kBuckets; b += kThreads) ws.parts[blockIdx.x * (int64_t)kBuckets + b] = hist.masses[b];
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_end_kernel(SampleArgs a, SampleSpace ws, int64_t chunks, int64_t chunk,
                                                             int shift) {
    __shared__ Shared sh;
    const int64_t at = blockIdx.x / chunks, c = blockIdx.x % chunks;
    const T *row = (const T *)a.logits + at * a.ld;
    const Settings s = settings_of(a, at);
    const uint64_t best = row_best(ws, at, chunks, sh.upart);
    if (settled(a, at, s, best, false)) return;
    const Row r = row_of(a, s, logit_of_key((uint32_t)(best >> 32)), shift);
    for (int b = threadIdx.x; b < kBuckets; b += kThreads)
        sh.hist.counts[b] = ws.counts[at * kBuckets + b], sh.hist.masses[b] = ws.masses[at * kBuckets + b];
    __syncthreads();
    const Plan p = plan_of(s, r, sh);
    const uint32_t room = (uint32_t)(chunk / 8);
    uint32_t *const list = ws.list + (at * chunks + c) * room;
    uint32_t placed = 0;
    if (p.hi >= 0)
        placed = collect(row, c * chunk, min((c + 1) * chunk, a.vocab), r, p, sh,
                         [&](uint32_t place, uint32_t index, uint32_t) {
                             if (place < room) put_shared(list + place, index);
                         });
    if (p.lo > 0 && s.masses) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kEach; i++) {
            const int b = threadIdx.x * kEach + i;
            if (b < p.lo) sum += (double)ws.parts[blockIdx.x * (int64_t)kBuckets + b] * p.unit[i];
        }
        sum = block_sum(sum, sh.part);
        if (threadIdx.x == 0) put_shared(ws.whole + blockIdx.x, sum);
    }
    if (threadIdx.x == 0) put_shared(ws.listed + blockIdx.x, placed);
    stores_arrived();
    __syncthreads();
    if (threadIdx.x == 0) sh.last = atomicAdd(&ws.done[at], 1u) == (uint32_t)chunks - 1;
    __syncthreads();
    if (!sh.last) return;
    // the chunks' lists in LDS, where they fit
    int64_t n = 0;
    bool fits = true;
    for (int64_t c0 = 0; c0 < chunks; c0 += kThreads) {
        const uint32_t mine = c0 + threadIdx.x < chunks ? get_shared(ws.listed + at * chunks + c0 + threadIdx.x) : 0;
        int64_t all;
        const int64_t upto = block_upto((int64_t)mine, sh.ipart, all);
        if (c0 == 0) sh.offset[threadIdx.x + 1] = (uint32_t)upto;
        if (c0 == 0 && threadIdx.x == 0) sh.offset[0] = 0;
        fits = block_max(mine > room, sh.upart) == 0 && fits;
        n += all;
    }
    __syncthreads();
    fits = fits && n <= kList && chunks <= kThreads;
    if (fits && n > 0) {
        // a thread finds the chunk of its place
        for (int i = threadIdx.x; i < n; i += kThreads) {
            int low = 0, high = (int)chunks;  // offset[low] <= i < offset[high]
            while (high - low > 1) {
                const int mid = (low + high) / 2;
                if (sh.offset[mid] <= (uint32_t)i)
                    low = mid;
                else
                    high = mid;
            }
            const uint32_t index = get_shared(ws.list + (at * chunks + low) * room + (i - sh.offset[low]));
            sh.index[i] = index;
            sh.key[i] = key_of(load_f32(row + index));
        }
        __syncthreads();
    }
    Kept kept = all_of(s, r, p);
    const bool ranked = fits && n > 0 && n <= kSorted;
    if (ranked) {
        if (by_rank(a, at, s, r, p, (int)n, sh, kept)) return;
    } else if (n > 0) {
        const Listed<T> l{row, r, p, sh, fits ? (int)n : -1};
        by_select(s, r, p, l, sh, kept);
        // the list's part of each chunk's mass
        if (fits) {
            const int lane = threadIdx.x % 64;
            for (int64_t w = threadIdx.x / 64; w < chunks; w += kWaves) {
                double sum = 0.0;
                for (uint32_t i = sh.offset[w] + lane; i < sh.offset[w + 1]; i += 64) {
                    const double x = r.x(logit_of_key(sh.key[i]));
                    if (kept.holds(sh.key[i], sh.index[i], x)) sum += mass(x);
                }
                sum = wave_sum(sum);
                if (lane == 0) {
                    double *const of = ws.whole + at * chunks + w;
                    put_shared(of, (p.lo > 0 && s.masses ? get_shared(of) : 0.0) + sum);
                }
            }
        } else {
            for (int64_t w = 0; w < chunks; w++) {
                double sum = 0.0;
                const int64_t end = min((w + 1) * chunk, a.vocab);
                for (int64_t t = w * chunk + threadIdx.x * 8; t < end; t += kTile) {
                    uint32_t k[8];
                    keys8(row, t, end, k);
#pragma unroll
                    for (int i = 0; i < 8; i++) {
                        if (!k[i]) continue;
                        const double x = r.x(logit_of_key(k[i]));
                        if (kept.holds(k[i], t + i, x)) sum += mass(x);
                    }
                }
                sum = block_sum(sum, sh.part);
                if (threadIdx.x == 0) put_shared(ws.whole + at * chunks + w, sum);
            }
        }
        stores_arrived();
        __syncthreads();
    }
    // the chunk whose tokens pass the drawn share, or the last that has any mass
    int64_t chosen = 0;
    double before = 0.0, start = 0.0;
    for (int64_t c0 = 0; c0 < chunks; c0 += kThreads) {
        const int64_t w = c0 + threadIdx.x;
        double m = w < chunks ? get_shared(ws.whole + at * chunks + w) : 0.0;
        if (ranked && w < chunks) m += sh.sorted.upto[sh.offset[w + 1]] - sh.sorted.upto[sh.offset[w]];
        double all;
        const double upto = before + block_upto(m, sh.part, all);
        const uint64_t hit = block_max(m > 0.0 && upto > kept.drawn ? kThreads - threadIdx.x : 0, sh.upart);
        const uint64_t any = hit ? 1 : block_max(m > 0.0 ? threadIdx.x + 1 : 0, sh.upart);
        if (any) {
            const int64_t owner = hit ? kThreads - (int64_t)hit : (int64_t)any - 1;
            if ((int64_t)threadIdx.x == owner) sh.value[0] = upto - m;
            chosen = c0 + owner;
            __syncthreads();
            start = sh.value[0];
            __syncthreads();
        }
        if (hit) break;
        before += all;
    }
    draw_in(a, at, row, r, kept, chosen * chunk, min((chosen + 1) * chunk, a.vocab), start, sh);
}

bool is_short(int64_t vocab) { return vocab <= kShort; }

template <typename T>
hipError_t sample_go(const SampleArgs &a, hipStream_t s) {
    int shift = 44;  // a bucket's mass, at most 2^shift for each token, fits 64 bits
    while (shift > 30 && a.vocab >> (63 - shift)) shift--;
    constexpr int64_t kStep = 1 << 22;  // workgroups of a launch, which holds fewer than 2^32 threads
    const int64_t chunk = chunk_of(a.rows, a.vocab), chunks = (a.vocab + chunk - 1) / chunk;
    const int64_t step = is_short(a.vocab) ? kStep : kStep / chunks;
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
        const unsigned grid = (unsigned)(is_short(a.vocab) ? p.rows : p.rows * chunks);
        if (is_short(a.vocab)) {
            sample_short_kernel<T><<<grid, kThreads, 0, s>>>(p, shift);
        } else {
            const SampleSpace ws = sample_space(a.ws, a.rows, a.vocab);
            sample_best_kernel<T><<<grid, kThreads, 0, s>>>(p, ws, chunks, chunk);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            sample_count_kernel<T><<<grid, kThreads, 0, s>>>(p, ws, chunks, chunk, shift);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            sample_end_kernel<T><<<grid, kThreads, 0, s>>>(p, ws, chunks, chunk, shift);
        }
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

size_t sample_workspace(int64_t rows, int64_t vocab) {
    return rows == 0 || is_short(vocab) ? 0 : sample_sizes(rows, vocab).bytes;
}

hipError_t launch_sample(const SampleArgs &a, bool bf16, hipStream_t stream) {
    if (a.rows == 0) return hipSuccess;
    return bf16 ? sample_go<__bf16>(a, stream) : sample_go<float>(a, stream);
}

}  // namespace sdnn
