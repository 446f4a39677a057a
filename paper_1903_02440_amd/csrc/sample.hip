// One winner per image drawn from its neurons' scores (gfx950).
//
// The order of the definition is that of the pairs (score from largest, index
// from smallest).  What steps 1 and 2 keep is a prefix of that order, so it is
// described by a boundary: every score above it, and the first `equal` indices
// of the scores equal to it.  A boundary is found on order-preserving 32-bit
// keys by histograms: of counts for top_k, of weights for top_p.  Weights are
// 64-bit fixed-point numbers, so that sums do not depend on the order of the
// histogram's atomics, nor of anything else.
//
// Rows of up to 16 keys a thread stay in registers.  Longer ones go through
// launches of several workgroups a row (largest score; histogram; the keys of the
// boundary's bin; sums by index; the draw), each reading the row again; where top_k
// keeps few, the list holds all that matters and the last two are one launch of
// a workgroup a row.  256 rows of 200003 floats: 32 us to read for the largest (6.4
// TB/s, in part from the cache behind HBM), 66 for the histogram of weights (36
// instructions a score), 37 for the list, 46 for the sums, 20 for the draw.  A row of
// 131072 bfloat16 scores, top_k 50: 4 + 5 + 8 + 10 us, the latency of four dependent
// steps.
#include <algorithm>
#include <cmath>

#include "common.hpp"
#include "libspyke_readout.h"

namespace {

struct SampleArgs {
    int64_t N;  // neurons of an image
    int T, HW, W, top_k, shift;  // shift: fraction bits of a weight
    float temperature, top_p, min_p;
};

template <class E>
__device__ __forceinline__ float as_float(E v);
template <>
__device__ __forceinline__ float as_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ float as_float<uint16_t>(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }

// Order-preserving key of a score; 0 for one that cannot win (NaN, -inf).
__device__ __forceinline__ uint32_t key_of(float v) {
    uint32_t b = __float_as_uint(v);
    b = b == 0x80000000u ? 0u : b;  // -0 and +0 are equal scores
    const uint32_t k = b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
    return v > -INFINITY ? k : 0u;  // (false for NaN)
}
__device__ __forceinline__ float value_of(uint32_t k) {
    return __uint_as_float(k ^ (k & 0x80000000u ? 0x80000000u : 0xFFFFFFFFu));
}

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) v += __shfl_xor(v, s, 64);
    return v;
}
__device__ __forceinline__ uint64_t wave_scan_u64(uint64_t v, int lane) {  // inclusive
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const uint64_t o = __shfl_up(v, s, 64);
        if (lane >= s) v += o;
    }
    return v;
}

constexpr int POW_BITS = 7, POW = 1 << POW_BITS;  // entries of the table of 2^(j / POW)
constexpr int BINS = 2048;  // bins of a row's first histogram
constexpr int LIST = 4096;  // keys of one bin that LDS takes

// Weights of a row: 2^shift exp((score - largest) / temperature), as integers.  With
// y = shift + (score - largest) log2(e) / temperature rounded to n + j / POW (by adding
// a number whose last place that is) and r what rounding left, it is 2^n 2^(j / POW)
// 2^r with 2^r from its series: the first term left out, (r ln 2)^5 / 120, is below
// 2e-15.  That and the roundings of y (2^-48) and of 1 / temperature (51 * 2^-53) stay
// below 1e-14 of the weight: eight steps of a weight near 2^51, less than one from
// shift 46 down.  +infinity as the largest weighs 2^shift.
struct Weigher {
    double top, per, shift_d;
    float ftop;
    const double *pow;
    __device__ __forceinline__ uint64_t operator()(uint32_t k) const { return of(value_of(k)); }
    __device__ __forceinline__ uint64_t of(float v) const {
        constexpr double LN2 = 0.69314718055994530942, STEP = 6755399441055744.0 / POW;  // 1.5 * 2^52 / POW
        const double d = v == ftop ? 0.0 : (double)v - top;
        const double y = fmax(fma(d, per, shift_d), -2.0);  // (below half: weight 0; NaN too)
        const double z = y + STEP;
        const int nj = (int)(uint32_t)__double_as_longlong(z);
        const double r = y - (z - STEP);
        double p = fma(r, LN2 * LN2 * LN2 * LN2 / 24, LN2 * LN2 * LN2 / 6);
        p = fma(r, p, LN2 * LN2 / 2);
        p = fma(r, p, LN2);
        p = fma(r, p, 1.0);
        const double w = ldexp(pow[nj & (POW - 1)] * p, nj >> POW_BITS);
        return (uint64_t)__double_as_longlong(w + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;  // (w < 2^52)
    }
};

constexpr int SHORT_BINS = 512;  // of a short row
constexpr int LONG_WAVES = 16, LONG_THREADS = LONG_WAVES * 64;

// LDS of a row's workgroup of WAVES waves.
template <int WAVES>
struct Shared {
    uint64_t hist[WAVES == LONG_WAVES ? BINS : SHORT_BINS];
    double pow[POW];
    uint64_t part[WAVES], part2[WAVES];
    uint64_t above;
    uint32_t bin, n_list;
    uint32_t list[WAVES == LONG_WAVES ? LIST : 64];
};

// Sum over the workgroup, in every thread.
template <int WAVES>
__device__ __forceinline__ uint64_t block_sum(Shared<WAVES> &sh, uint64_t v) {
    v = wave_sum_u64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.part[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t s = 0;
#pragma unroll
    for (int q = 0; q < WAVES; ++q) s += sh.part[q];
    return s;
}

// The first of N bins (from bin 0) at which the running total reaches `want`,
// the last one if it never does; *above gets the total of the bins before it.
template <int N, int WAVES>
__device__ __forceinline__ uint32_t find_bin(Shared<WAVES> &sh, uint64_t want, uint64_t *above) {
    constexpr int THREADS = WAVES * 64, PER = N < THREADS ? 1 : N / THREADS, USED = N / PER;  // bins of a thread
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    __syncthreads();
    uint64_t v[PER], sum = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        v[j] = tid < USED ? sh.hist[tid * PER + j] : 0;
        sum += v[j];
    }
    const uint64_t incl = wave_scan_u64(sum, lane);
    if (lane == 63) sh.part[wv] = incl;
    __syncthreads();
    uint64_t run = incl - sum;
#pragma unroll
    for (int q = 0; q < WAVES; ++q) run += q < wv ? sh.part[q] : 0;
    if (run < want && (run + sum >= want || tid == USED - 1) && tid < USED) {
        int at = PER - 1;
        bool found = false;
#pragma unroll
        for (int j = 0; j < PER - 1; ++j) {
            if (!found && run + v[j] >= want) {
                at = j;
                found = true;
            }
            run += found ? 0 : v[j];
        }
        sh.bin = (uint32_t)(tid * PER + at);
        sh.above = run;
    }
    __syncthreads();
    *above = sh.above;
    return sh.bin;
}

// The key at which the running total of value(k), from the largest key, reaches
// `want` among the n <= 64 keys of the list that are not below `from`: a key a
// lane, each against all.  *above_edge gets the total of the larger keys.
template <int WAVES, class Value>
__device__ __forceinline__ uint32_t few(Shared<WAVES> &sh, uint32_t n, uint32_t from, uint64_t want, Value value,
                                        uint64_t *above_edge) {
    __syncthreads();
    if (threadIdx.x < 64) {
        const uint32_t x = threadIdx.x < n ? sh.list[threadIdx.x] : 0, k = x >= from ? x : 0;
        const uint64_t v = k ? value(k) : 0;
        uint64_t above = 0, equal = 0;
        for (uint32_t j = 0; j < n; ++j) {
            const uint32_t kj = (uint32_t)__builtin_amdgcn_readlane((int)k, (int)j);
            const uint64_t vj = ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), (int)j) << 32) |
                                (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, (int)j);
            above += kj > k ? vj : 0;
            equal += kj == k ? vj : 0;
        }
        if (k && above < want && want <= above + equal) {  // (equal keys write the same)
            sh.bin = k;
            sh.above = above;
        }
    }
    __syncthreads();
    *above_edge = sh.above;
    return sh.bin;
}

// As few() for n up to a thread a key, the values in the histogram's room.
template <int WAVES, class Value>
__device__ __forceinline__ uint32_t some(Shared<WAVES> &sh, uint32_t n, uint32_t from, uint64_t want, Value value,
                                         uint64_t *above_edge) {
    static_assert(WAVES == LONG_WAVES && LONG_THREADS <= BINS && LONG_THREADS <= LIST, "a place a thread");
    const uint32_t x = threadIdx.x < n ? sh.list[threadIdx.x] : 0, k = x >= from ? x : 0;
    __syncthreads();
    sh.list[threadIdx.x] = k;
    sh.hist[threadIdx.x] = k ? value(k) : 0;
    __syncthreads();
    if (k) {
        uint64_t above = 0, equal = 0;
        for (uint32_t j = 0; j < n; j += 8) {  // (behind n: keys 0)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t kj = sh.list[j + i];
                const uint64_t vj = sh.hist[j + i];
                above += kj > k ? vj : 0;
                equal += kj == k ? vj : 0;
            }
        }
        if (above < want && want <= above + equal) {  // (equal keys write the same)
            sh.bin = k;
            sh.above = above;
        }
    }
    __syncthreads();
    *above_edge = sh.above;
    return sh.bin;
}

// The key at which the running total of the values, from the largest key, reaches
// `want` among the keys that each(f) calls f(key, value()) with; its four digits
// in turn.  *above_edge gets the total of the larger keys.
template <int WAVES, class Each>
__device__ __forceinline__ uint32_t descend(Shared<WAVES> &sh, uint64_t want, Each each, uint64_t *above_edge) {
    uint32_t prefix = 0;
    uint64_t above = 0;
    for (int sft = 24; sft >= 0; sft -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += WAVES * 64) sh.hist[i] = 0;
        __syncthreads();
        each([&](uint32_t k, auto value) {
            if (sft == 24 || (k >> (sft + 8)) == prefix) {
                const uint64_t v = value();
                if (v) atomicAdd((unsigned long long *)&sh.hist[255 - ((k >> sft) & 255)], (unsigned long long)v);
            }
        });
        uint64_t over;
        const uint32_t bin = find_bin<256, WAVES>(sh, want - above, &over);
        prefix = (prefix << 8) | (255 - bin);
        above += over;
    }
    *above_edge = above;
    return prefix;
}

// A row's boundary: keys above `edge` stay, and the first `equal` of those equal to it.
struct Edge {
    uint32_t edge = 1;
    uint64_t equal = ~0ull;
    __device__ __forceinline__ void by_weight(uint32_t e, uint64_t want, uint64_t above, uint64_t we) {
        const uint64_t m = we ? (want - above + we - 1) / we : 1;
        equal = e == edge ? (m < equal ? m : equal) : m;
        edge = e;
    }
};

// top_p's share of a sum
__device__ __forceinline__ uint64_t share(float top_p, uint64_t sum) {
    const uint64_t want = (uint64_t)ceil((double)top_p * (double)sum);
    return want < 1 ? 1 : (want > sum ? sum : want);
}

__device__ __forceinline__ uint64_t target_of(float u, uint64_t all) {
    const uint64_t t = (uint64_t)((u > 0.0f ? fmin((double)u, 1.0) : 0.0) * (double)all);
    return t < all ? t : all - 1;
}

__device__ __forceinline__ void put_winner(int32_t *winners, int32_t *n_win, int64_t b, int64_t n, int t,
                                           const SampleArgs &a) {
    winners[b * 4 + 0] = (int32_t)(n / a.HW);
    winners[b * 4 + 1] = t;
    winners[b * 4 + 2] = (int32_t)(n % a.HW / a.W);
    winners[b * 4 + 3] = (int32_t)(n % a.HW % a.W);
    n_win[b] = 1;
}

template <int WAVES>
__device__ __forceinline__ Weigher weigher(Shared<WAVES> &sh, const SampleArgs &a, uint32_t ktop) {
    for (int i = threadIdx.x; i < POW; i += WAVES * 64) sh.pow[i] = exp2(i * (1.0 / POW));
    Weigher w;
    w.top = (double)value_of(ktop);
    w.per = a.temperature > 0.0f ? 1.4426950408889634074 / (double)a.temperature : 0.0;
    w.ftop = value_of(ktop);
    w.shift_d = (double)a.shift;
    w.pow = sh.pow;
    return w;
}

// Sums over the threads before this one, and over all.
template <int WAVES>
__device__ __forceinline__ void before_and_all(Shared<WAVES> &sh, uint64_t x, uint64_t y, uint64_t *xb, uint64_t *yb,
                                               uint64_t *xa, uint64_t *ya) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    const uint64_t xi = wave_scan_u64(x, lane), yi = wave_scan_u64(y, lane);
    __syncthreads();
    if (lane == 63) {
        sh.part[wv] = xi;
        sh.part2[wv] = yi;
    }
    __syncthreads();
    *xb = xi - x, *yb = yi - y, *xa = 0, *ya = 0;
    for (int q = 0; q < WAVES; ++q) {
        *xb += q < wv ? sh.part[q] : 0;
        *yb += q < wv ? sh.part2[q] : 0;
        *xa += sh.part[q];
        *ya += sh.part2[q];
    }
}

// The draw among `n` keys of a thread that follow each other in index (0 =
// cannot win): keys above the edge and the first `equal` equal to it, of weight
// min_w at least.  key_at(i) gives the thread's i-th key.  `run`, `eq`: kept weight and equal keys before the workgroup's first.
// Returns whether this thread holds the winner, and its number.
template <int WAVES, class KeyAt>
__device__ __forceinline__ bool pick(Shared<WAVES> &sh, const Weigher &weigh, uint64_t we, const Edge &e, uint64_t min_w, uint64_t target,
                                     uint64_t run, uint64_t eq, int64_t n, KeyAt key_at, int64_t *at) {
    constexpr int AHEAD = 8;  // keys read at a time
    uint64_t sum = 0, eqs = 0;
    for (int64_t i = 0; i < n; i += AHEAD) {
        uint32_t k[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) k[j] = key_at(min(i + j, n - 1));
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (i + j >= n) continue;
            const uint64_t w = k[j] > e.edge ? weigh(k[j]) : 0;
            sum += w >= min_w ? w : 0;
            eqs += k[j] == e.edge;
        }
    }
    uint64_t run_in, eq_in, all, eq_all;
    before_and_all<WAVES>(sh, sum, eqs, &run_in, &eq_in, &all, &eq_all);
    run += run_in;
    eq += eq_in;
    // kept weight before this thread, equal keys among it
    const uint64_t before = run + (eq < e.equal ? eq : e.equal) * we;
    const uint64_t left = eq < e.equal ? e.equal - eq : 0;
    const uint64_t own = sum + (eqs < left ? eqs : left) * we;
    if (!(target >= before && target < before + own)) return false;
    uint64_t r = before, l = left;
    for (int64_t i = 0; i < n; ++i) {
        const uint32_t k = key_at(i);
        uint64_t w = 0;
        if (k > e.edge) {
            w = weigh(k);
            w = w >= min_w ? w : 0;
        } else if (k == e.edge && l) {
            w = we;
            --l;
        }
        r += w;
        if (r > target) {
            *at = i;
            return true;
        }
    }
    return false;  // (not reached)
}

// Bins of a row's histogram: equal steps of the score from the largest down to
// the smallest, or to where weights end (44 temperatures); the last bin takes the rest.
struct Bins {
    float top, steps, last;
    __device__ __forceinline__ Bins(float hi, float lo, float temperature, int n)
        : top(hi), steps((float)(n - 2) / fmaxf(fminf(hi - lo, 44.0f * temperature), 1e-30f)), last((float)(n - 1)) {}
    __device__ __forceinline__ int operator()(float v) const {  // does not fall as the score falls
        return v == top ? 0 : (int)fminf((top - v) * steps, last);
    }
};

// As descend(), by a histogram of SHORT_BINS bins first and then the boundary's
// bin alone, whose keys are few as a rule.
template <int WAVES, class Each, class Value>
__device__ __forceinline__ uint32_t boundary(Shared<WAVES> &sh, const Bins &bins, uint32_t from, uint64_t want, Each each,
                                             Value value, uint64_t *above_edge) {
    __syncthreads();
    for (int i = threadIdx.x; i < SHORT_BINS; i += WAVES * 64) sh.hist[i] = 0;
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
    each([&](uint32_t k, auto v) {
        atomicAdd((unsigned long long *)&sh.hist[bins(value_of(k))], (unsigned long long)v());
    });
    uint64_t over, in;
    const int bin = (int)find_bin<SHORT_BINS, WAVES>(sh, want, &over);
    each([&](uint32_t k, auto) {
        if (bins(value_of(k)) == bin) {
            const uint32_t at = atomicAdd(&sh.n_list, 1u);
            if (at < 64) sh.list[at] = k;
        }
    });
    __syncthreads();
    const uint32_t n = sh.n_list;
    const uint32_t key = n <= 64 ? few<WAVES>(sh, n, from, want - over, value, &in)
                                 : descend<WAVES>(sh, want - over, [&](auto f) {
                                       each([&](uint32_t k, auto v) {
                                           if (bins(value_of(k)) == bin) f(k, v);
                                       });
                                   }, &in);
    *above_edge = over + in;
    return key;
}

// Grid: one workgroup per image, whose row of at most 16 keys a thread stays in
// registers; a thread's keys follow each other in index.  Read once; bound by the
// chain of short steps between barriers (1000 masked images of 200x4x4 in 21 us,
// 0.8 TB/s; a single image 10).
template <class E, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 4) void k_sample_short(const E *__restrict__ scores,
                                                             const uint8_t *__restrict__ t_first,
                                                             const float *__restrict__ u, SampleArgs a,
                                                             int32_t *__restrict__ winners,
                                                             int32_t *__restrict__ n_win) {
    constexpr int KEYS = 16;
    __shared__ Shared<WAVES> sh;
    const int tid = threadIdx.x;
    const int64_t b = blockIdx.x;
    const int N = (int)a.N, per = (N + WAVES * 64 - 1) / (WAVES * 64), i0 = tid * per;
    const E *x = scores + b * a.N;
    const uint8_t *tf = t_first ? t_first + b * a.N : nullptr;
    uint32_t key[KEYS];
    E raw[KEYS];
#pragma unroll
    for (int j = 0; j < KEYS; ++j) raw[j] = x[min(i0 + min(j, per - 1), N - 1)];
    if (tf) {
        uint8_t t[KEYS];
#pragma unroll
        for (int j = 0; j < KEYS; ++j) t[j] = tf[min(i0 + min(j, per - 1), N - 1)];
#pragma unroll
        for (int j = 0; j < KEYS; ++j) key[j] = t[j] < a.T ? key_of(as_float<E>(raw[j])) : 0u;
    } else {
#pragma unroll
        for (int j = 0; j < KEYS; ++j) key[j] = key_of(as_float<E>(raw[j]));
    }
    uint32_t hi = 0, low = 0;  // largest and (of ~key) smallest key that can win
    uint64_t cnt = 0;
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
        key[j] = j < per && i0 + j < N ? key[j] : 0u;
        hi = max(hi, key[j]);
        low = max(low, key[j] ? ~key[j] : 0u);
        cnt += key[j] != 0;
    }
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) {
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, s, 64));
        low = max(low, (uint32_t)__shfl_xor((int)low, s, 64));
    }
    if ((tid & 63) == 0) sh.part2[tid >> 6] = ((uint64_t)hi << 32) | low;
    const uint64_t total = block_sum<WAVES>(sh, cnt);
#pragma unroll
    for (int q = 0; q < WAVES; ++q) {
        hi = max(hi, (uint32_t)(sh.part2[q] >> 32));
        low = max(low, (uint32_t)sh.part2[q]);
    }
    const uint32_t top = hi;
    if (top == 0) {  // nothing can win (uniform)
        if (tid < 4) winners[b * 4 + tid] = -1;
        if (tid == 0) n_win[b] = 0;
        return;
    }
    const Weigher weigh = weigher<WAVES>(sh, a, top);
    const Bins bins(value_of(top), value_of(~low), a.temperature, SHORT_BINS);
    __syncthreads();
    Edge e;
    uint64_t above;
    const uint64_t top_k = a.temperature > 0.0f ? (uint64_t)a.top_k : 1ull;
    if (top_k == 1) {
        e.edge = top;
        e.equal = 1;
    } else if (top_k > 0 && top_k < total) {
        e.edge = boundary<WAVES>(sh, bins, 1, top_k, [&](auto f) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
                if (key[j]) f(key[j], [] { return (uint64_t)1; });
        }, [](uint32_t) { return (uint64_t)1; }, &above);
        e.equal = top_k - above;
    }
    uint64_t w[KEYS];
#pragma unroll
    for (int j = 0; j < KEYS; ++j) w[j] = key[j] >= e.edge ? weigh(key[j]) : 0;
    if (a.top_p < 1.0f && top_k != 1) {
        uint64_t sum = 0;
#pragma unroll
        for (int j = 0; j < KEYS; ++j) sum += key[j] > e.edge || e.equal == ~0ull ? w[j] : 0;
        sum = block_sum<WAVES>(sh, sum);
        if (e.equal != ~0ull) sum += e.equal * weigh(e.edge);
        const uint64_t want = share(a.top_p, sum);
        // (the edge of step 1 takes part with all its equals: one that step 1 cut has its own limit)
        const uint32_t k = boundary<WAVES>(sh, bins, e.edge, want, [&](auto f) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
                if (w[j]) f(key[j], [&] { return w[j]; });
        }, weigh, &above);
        e.by_weight(k, want, above, weigh(k));
    }
    const uint64_t min_w = (uint64_t)ceil(ldexp((double)a.min_p, a.shift));
    // the sum of what is left, and the draw
    uint64_t we = weigh(e.edge), sum = 0, eqs = 0;
    we = we >= min_w ? we : 0;
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
        w[j] = key[j] > e.edge && w[j] >= min_w ? w[j] : 0;
        sum += w[j];
        eqs += key[j] == e.edge;
    }
    uint64_t run, eq, all, eq_all;
    before_and_all<WAVES>(sh, sum, eqs, &run, &eq, &all, &eq_all);
    const uint64_t target = target_of(u[b], all + (eq_all < e.equal ? eq_all : e.equal) * we);
    // the thread that holds the target walks its keys
    uint64_t left = e.equal - (eq < e.equal ? eq : e.equal);
    run += (eq < e.equal ? eq : e.equal) * we;
    if (!(target >= run && target < run + sum + (eqs < left ? eqs : left) * we)) return;
    int at = -1;
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
        const bool is_edge = key[j] == e.edge && left > 0;
        left -= is_edge;
        run += w[j] + (is_edge ? we : 0);
        at = at < 0 && run > target ? j : at;
    }
    put_winner(winners, n_win, b, i0 + at, tf ? (int)tf[i0 + at] : 0, a);
}

constexpr int SPLITS = 64;  // workgroups of a row at most

// Calls f(score, index) for the indices i0 <= index < i1 of a row, by `threads`
// threads of which this is number `t`: vectors of 16 bytes, four in flight a
// thread, and the ends that no whole vector covers one by one.  A masked score
// is -infinity.
template <class E, class F>
__device__ __forceinline__ void for_row(const E *x, const uint8_t *tf, int T, int64_t i0, int64_t i1, int t, int threads,
                                        F f) {
    constexpr int V = 16 / sizeof(E), UNR = 4;
    const int64_t skip = (V - (int64_t)((reinterpret_cast<uintptr_t>(x + i0) / sizeof(E)) % V)) % V;
    const int64_t v0 = min(i1, i0 + skip);
    const int nv = (int)((i1 - v0) / V);
    struct alignas(16) Vec {
        E e[V];
    };
    const Vec *xv = reinterpret_cast<const Vec *>(x + v0);
    for (int j = t; j < nv; j += threads * UNR) {
        Vec r[UNR];
        uint8_t tt[UNR][V];
#pragma unroll
        for (int q = 0; q < UNR; ++q) r[q] = xv[min(j + q * threads, nv - 1)];
        if (tf) {
#pragma unroll
            for (int q = 0; q < UNR; ++q)
#pragma unroll
                for (int c = 0; c < V; ++c) tt[q][c] = tf[v0 + (int64_t)min(j + q * threads, nv - 1) * V + c];
        }
#pragma unroll
        for (int q = 0; q < UNR; ++q) {
            if (j + q * threads >= nv) break;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                const float v = as_float<E>(r[q].e[c]);
                f(tf && tt[q][c] >= T ? -INFINITY : v, v0 + (int64_t)(j + q * threads) * V + c);
            }
        }
    }
    const int64_t head = v0 - i0, tail = i1 - v0 - (int64_t)nv * V;  // below V each
    if (t < head + tail) {
        const int64_t i = t < head ? i0 + t : i1 - tail + (t - head);
        const float v = as_float<E>(x[i]);
        f(tf && tf[i] >= T ? -INFINITY : v, i);
    }
}

// Workspace of long rows: each step is a launch of `splits` workgroups a row.
struct RowPart {
    float top, low;  // largest and smallest score that can win
    uint32_t n;      // how many can
};
struct RowSums {
    uint64_t kept, equal;  // weight above the edge, keys equal to it
};
struct RowEdge {
    uint64_t equal;
    uint32_t edge, any;
};
struct Work {
    int splits;
    uint64_t *hist;   // [B][BINS]
    uint64_t *list;   // [B][LIST], entries
    uint32_t *count;  // [B]
    RowPart *part;    // [B][splits]
    RowSums *sums;    // [B][splits][LONG_WAVES]
    RowEdge *edge;    // [B]
};

// A score in a list: larger where it comes earlier in the order.
__device__ __forceinline__ uint64_t entry(uint32_t key, int64_t i) { return ((uint64_t)key << 32) | (uint32_t)~(uint32_t)i; }

// A long row's scores and the workgroup's share of them.
template <class E>
struct LongRow {
    const E *x;
    const uint8_t *tf;
    int64_t N, i0, i1, seg;
    int T;
    __device__ __forceinline__ LongRow(const E *scores, const uint8_t *t_first, const SampleArgs &a, int splits, int64_t b,
                                       int split)
        : x(scores + b * a.N), tf(t_first ? t_first + b * a.N : nullptr), N(a.N), T(a.T) {
        seg = ((N + (int64_t)splits * LONG_WAVES - 1) / ((int64_t)splits * LONG_WAVES) + 7) / 8 * 8;  // of a wave
        i0 = min(N, split * LONG_WAVES * seg);
        i1 = min(N, i0 + LONG_WAVES * seg);
    }
    template <class F>
    __device__ __forceinline__ void own(F f) const { for_row<E>(x, tf, T, i0, i1, threadIdx.x, LONG_THREADS, f); }
    template <class F>
    __device__ __forceinline__ void all(F f) const { for_row<E>(x, tf, T, 0, N, threadIdx.x, LONG_THREADS, f); }
    // f(key, value()) for the row's keys from the edge up
    template <class F, class Value>
    __device__ __forceinline__ void each_from(const Edge &from, F f, Value value) const {
        all([&](float v, int64_t) {
            const uint32_t k = key_of(v);
            if (k >= from.edge && k != 0) f(k, [&] { return value(k); });
        });
    }
};

// What a row's parts add up to, and the bins of its histogram.
struct RowStat {
    float top, low;
    uint32_t n;
    Bins bin;
    __device__ __forceinline__ RowStat(const RowPart *part, int splits, float temperature)
        : RowStat(total(part, splits), temperature) {}

  private:
    __device__ __forceinline__ RowStat(const RowPart &p, float temperature)
        : top(p.top), low(p.low), n(p.n), bin(p.top, p.low, temperature, BINS) {}
    static __device__ __forceinline__ RowPart total(const RowPart *part, int splits) {
        const int lane = threadIdx.x & 63;
        RowPart p = part[min(lane, splits - 1)];
        int m = lane < splits ? (int)p.n : 0;
#pragma unroll
        for (int s = 32; s >= 1; s >>= 1) {
            p.top = fmaxf(p.top, __shfl_xor(p.top, s, 64));
            p.low = fminf(p.low, __shfl_xor(p.low, s, 64));
            m += __shfl_xor(m, s, 64);
        }
        p.n = (uint32_t)m;
        return p;
    }
};

__device__ __forceinline__ bool wins(float v) { return v > -INFINITY; }  // (false for NaN)

template <class E>
__global__ __launch_bounds__(LONG_THREADS) void k_sample_top(const E *__restrict__ scores,
                                                             const uint8_t *__restrict__ t_first, SampleArgs a, Work w) {
    __shared__ RowPart sh[LONG_WAVES];
    const int64_t b = blockIdx.y;
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    for (int i = blockIdx.x * LONG_THREADS + threadIdx.x; i < BINS; i += gridDim.x * LONG_THREADS) w.hist[b * BINS + i] = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) w.count[b] = 0;
    const LongRow<E> row(scores, t_first, a, w.splits, b, blockIdx.x);
    float hi = -INFINITY, lo = INFINITY;
    int n = 0;
    row.own([&](float v, int64_t) {
        hi = fmaxf(hi, v);  // (the other one where one is NaN)
        lo = fminf(lo, wins(v) ? v : INFINITY);
        n += wins(v);
    });
#pragma unroll
    for (int s = 32; s >= 1; s >>= 1) {
        hi = fmaxf(hi, __shfl_xor(hi, s, 64));
        lo = fminf(lo, __shfl_xor(lo, s, 64));
        n += __shfl_xor(n, s, 64);
    }
    if (lane == 0) sh[wv] = RowPart{hi, lo, (uint32_t)n};
    __syncthreads();
    if (threadIdx.x == 0) {
        RowPart p = sh[0];
        for (int q = 1; q < LONG_WAVES; ++q) {
            p.top = fmaxf(p.top, sh[q].top);
            p.low = fminf(p.low, sh[q].low);
            p.n += sh[q].n;
        }
        w.part[b * w.splits + blockIdx.x] = p;
    }
}

// The row's histogram, of counts or of weights.
template <class E, bool COUNT>
__global__ __launch_bounds__(LONG_THREADS) void k_sample_hist(const E *__restrict__ scores,
                                                              const uint8_t *__restrict__ t_first, SampleArgs a, Work w) {
    __shared__ Shared<LONG_WAVES> sh;
    const int64_t b = blockIdx.y;
    const RowStat st(w.part + b * w.splits, w.splits, a.temperature);
    if (st.n == 0) return;
    const Weigher weigh = weigher<LONG_WAVES>(sh, a, key_of(st.top));
    for (int i = threadIdx.x; i < BINS; i += LONG_THREADS) sh.hist[i] = 0;
    __syncthreads();
    const LongRow<E> row(scores, t_first, a, w.splits, b, blockIdx.x);
    row.own([&](float v, int64_t) {
        const uint64_t x = COUNT ? 1 : weigh.of(v);
        if (wins(v) && x) atomicAdd((unsigned long long *)&sh.hist[st.bin(v)], (unsigned long long)x);
    });
    __syncthreads();
    for (int i = threadIdx.x; i < BINS; i += LONG_THREADS)
        if (sh.hist[i]) atomicAdd((unsigned long long *)&w.hist[b * BINS + i], (unsigned long long)sh.hist[i]);
}

// The boundary's bin of the row's histogram and what lies before it.
template <bool COUNT>
__device__ __forceinline__ int boundary_bin(Shared<LONG_WAVES> &sh, const SampleArgs &a, const Work &w, int64_t b,
                                            uint64_t *want, uint64_t *over) {
    uint64_t sum = 0;
    for (int i = threadIdx.x; i < BINS; i += LONG_THREADS) sum += sh.hist[i] = w.hist[b * BINS + i];
    sum = block_sum<LONG_WAVES>(sh, sum);
    *want = COUNT ? (uint64_t)a.top_k : share(a.top_p, sum);
    return (int)find_bin<BINS, LONG_WAVES>(sh, *want, over);
}

// The entries of the boundary's bin; with COUNT those of the bins before it too,
// so that what step 1 keeps is all there.
template <class E, bool COUNT>
__global__ __launch_bounds__(LONG_THREADS) void k_sample_list(const E *__restrict__ scores,
                                                              const uint8_t *__restrict__ t_first, SampleArgs a, Work w) {
    __shared__ Shared<LONG_WAVES> sh;
    __shared__ uint64_t list[LIST];
    const int64_t b = blockIdx.y;
    const RowStat st(w.part + b * w.splits, w.splits, a.temperature);
    if (st.n == 0) return;
    uint64_t want, over;
    const int bin = boundary_bin<COUNT>(sh, a, w, b, &want, &over);
    const LongRow<E> row(scores, t_first, a, w.splits, b, blockIdx.x);
    if (threadIdx.x == 0) sh.n_list = 0;
    __syncthreads();
    row.own([&](float v, int64_t i) {
        if (!wins(v)) return;
        const int at_bin = st.bin(v);
        if (at_bin == bin || (COUNT && at_bin < bin)) {
            const uint32_t at = atomicAdd(&sh.n_list, 1u);
            if (at < LIST) list[at] = entry(key_of(v), i);
        }
    });
    __syncthreads();
    const uint32_t n = sh.n_list;  // (beyond LIST the row goes without its list)
    if (threadIdx.x == 0) sh.bin = n ? atomicAdd(&w.count[b], n) : 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x, at = sh.bin; i < n && i < LIST; i += LONG_THREADS)
        if (at + i < LIST) w.list[b * LIST + at + i] = list[i];
}

// The smallest score that can weigh min_w (some lower ones pass too).
__device__ __forceinline__ float least(const SampleArgs &a, float top, uint64_t min_w) {
    if (min_w <= 1) return -INFINITY;
    const double d = (double)a.temperature * (log(ldexp((double)(min_w - 1), -a.shift)) - 1e-6);  // (at most 0)
    const double v = (double)top + d;
    return nextafterf((float)v, -INFINITY);
}

// Step 1's boundary, then step 2's, among the keys that each(e, f, value) calls
// f(key, value()) with, those from the edge e up; the `n` of the list, if they are
// few, lie in sh.list.
template <class Each>
__device__ __forceinline__ Edge edge_of_count(Shared<LONG_WAVES> &sh, const SampleArgs &a, const Weigher &weigh, uint32_t n,
                                              uint32_t total, Each each) {
    constexpr int WAVES = LONG_WAVES;
    auto one = [](uint32_t) { return (uint64_t)1; };
    Edge e;
    uint64_t above;
    if ((uint64_t)a.top_k < total) {
        const uint32_t k = n <= WAVES * 64 ? some<WAVES>(sh, n, e.edge, (uint64_t)a.top_k, one, &above)
                                           : descend<WAVES>(sh, (uint64_t)a.top_k, [&](auto f) { each(e, f, one); }, &above);
        e.equal = (uint64_t)a.top_k - above;
        e.edge = k;
    }
    if (a.top_p < 1.0f) {
        uint64_t sum = 0;
        each(e, [&](uint32_t k, auto value) {
            if (k > e.edge || e.equal == ~0ull) sum += value();
        }, weigh);
        sum = block_sum<WAVES>(sh, sum);
        if (e.equal != ~0ull) sum += e.equal * weigh(e.edge);
        const uint64_t want = share(a.top_p, sum);
        // (the edge takes part with all its equals: one that step 1 cut has its own limit)
        const uint32_t k = n <= WAVES * 64 ? some<WAVES>(sh, n, e.edge, want, weigh, &above)
                                           : descend<WAVES>(sh, want, [&](auto f) { each(e, f, weigh); }, &above);
        e.by_weight(k, want, above, weigh(k));
    }
    return e;
}

// The boundary (each workgroup of the row finds it for itself), then the sums of
// the waves' segments.  FORM: 0 nothing is cut, or all but the largest; 1 by
// weight; 2 by count, then by weight.
template <class E, int FORM>
__global__ __launch_bounds__(LONG_THREADS) void k_sample_sums(const E *__restrict__ scores,
                                                              const uint8_t *__restrict__ t_first, SampleArgs a, Work w) {
    constexpr int WAVES = LONG_WAVES;
    __shared__ Shared<WAVES> sh;
    const int64_t b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const RowStat st(w.part + b * w.splits, w.splits, a.temperature);
    if (st.n == 0) {
        if (blockIdx.x == 0 && tid == 0) w.edge[b].any = 0;
        return;
    }
    const uint32_t ktop = key_of(st.top);
    const Weigher weigh = weigher<WAVES>(sh, a, ktop);
    const LongRow<E> row(scores, t_first, a, w.splits, b, blockIdx.x);
    __syncthreads();
    Edge e;
    if (FORM == 0) {
        if (a.temperature == 0.0f || a.top_k == 1) {
            e.edge = ktop;
            e.equal = 1;
        }
    } else {
        uint64_t want = 0, over = 0, above;
        if (FORM == 1) boundary_bin<false>(sh, a, w, b, &want, &over);
        const uint32_t n = w.count[b];
        const bool listed = n <= LIST;
        if (listed) {
            for (uint32_t i = tid; i < n; i += LONG_THREADS) sh.list[i] = (uint32_t)(w.list[b * LIST + i] >> 32);
            __syncthreads();
        }
        // f(key, value()) for the keys from the edge up: of the list, else of the whole row
        auto each = [&](const Edge &from, auto f, auto value) {
            if (listed) {
                for (uint32_t i = tid; i < n; i += LONG_THREADS) {
                    const uint32_t k = sh.list[i];
                    if (k >= from.edge) f(k, [&] { return value(k); });
                }
            } else {
                row.each_from(from, f, value);
            }
        };
        if (FORM == 1) {
            // (the list is the boundary's bin alone; the row stands for all bins)
            const uint64_t rest = listed ? want - over : want;
            const uint32_t k = n <= WAVES * 64 ? some<WAVES>(sh, n, e.edge, rest, weigh, &above)
                                               : descend<WAVES>(sh, rest, [&](auto f) { each(e, f, weigh); }, &above);
            e.by_weight(k, rest, above, weigh(k));
        } else {
            e = edge_of_count(sh, a, weigh, n, st.n, each);
        }
    }
    const uint64_t min_w = (uint64_t)ceil(ldexp((double)a.min_p, a.shift));
    const float edge = e.edge > 1 ? value_of(e.edge) : -INFINITY;  // (1: everything that can win is above)
    const float low = least(a, st.top, min_w);
    uint64_t sum = 0;
    uint32_t eqs = 0;
    const int64_t s0 = min(row.i1, row.i0 + wv * row.seg), s1 = min(row.i1, s0 + row.seg);
    for_row<E>(row.x, row.tf, row.T, s0, s1, lane, 64, [&](float v, int64_t) {
        if (v > edge && v >= low) {
            const uint64_t x = weigh.of(v);
            sum += x >= min_w ? x : 0;
        }
        eqs += v == edge && wins(v);
    });
    sum = wave_sum_u64(sum);
    const uint64_t eqn = wave_sum_u64(eqs);
    if (lane == 0) w.sums[(b * w.splits + blockIdx.x) * WAVES + wv] = RowSums{sum, eqn};
    if (blockIdx.x == 0 && tid == 0) w.edge[b] = RowEdge{e.equal, e.edge, 1};
}

// Grid: one workgroup per row: the segment of the draw, then the winner in it.
template <class E>
__global__ __launch_bounds__(LONG_THREADS) void k_sample_pick(const E *__restrict__ scores,
                                                              const uint8_t *__restrict__ t_first,
                                                              const float *__restrict__ u, SampleArgs a, Work w,
                                                              int32_t *__restrict__ winners,
                                                              int32_t *__restrict__ n_win) {
    constexpr int WAVES = LONG_WAVES;
    __shared__ Shared<WAVES> sh;
    const int64_t b = blockIdx.x;
    const int tid = threadIdx.x;
    const RowEdge re = w.edge[b];
    if (!re.any) {  // nothing can win (uniform)
        if (tid < 4) winners[b * 4 + tid] = -1;
        if (tid == 0) n_win[b] = 0;
        return;
    }
    const RowStat st(w.part + b * w.splits, w.splits, a.temperature);
    const Weigher weigh = weigher<WAVES>(sh, a, key_of(st.top));
    const int ns = w.splits * WAVES;
    __syncthreads();
    Edge e;
    e.edge = re.edge;
    e.equal = re.equal;
    const uint64_t min_w = (uint64_t)ceil(ldexp((double)a.min_p, a.shift));
    uint64_t we = e.edge > 1 ? weigh(e.edge) : 0;
    we = we >= min_w ? we : 0;
    // kept weight and equal keys before each segment (a thread a segment)
    const RowSums own = tid < ns ? w.sums[b * ns + tid] : RowSums{0, 0};
    uint64_t run, eq, all, eq_all;
    before_and_all<WAVES>(sh, own.kept, own.equal, &run, &eq, &all, &eq_all);
    const uint64_t target = target_of(u[b], all + (eq_all < e.equal ? eq_all : e.equal) * we);
    const uint64_t used = eq < e.equal ? eq : e.equal, left = e.equal - used;
    const uint64_t before = run + used * we, mine = own.kept + (own.equal < left ? own.equal : left) * we;
    if (target >= before && target < before + mine) {
        sh.bin = (uint32_t)tid;
        sh.above = run;
        sh.hist[0] = eq;
    }
    __syncthreads();
    const int at_seg = (int)sh.bin;
    run = sh.above;
    eq = sh.hist[0];
    const LongRow<E> row(scores, t_first, a, w.splits, b, at_seg / WAVES);
    const int64_t g0 = min(row.i1, row.i0 + (at_seg % WAVES) * row.seg), g1 = min(row.i1, g0 + row.seg);
    const int64_t per = (g1 - g0 + LONG_THREADS - 1) / LONG_THREADS;
    const int64_t i0 = min(g1, g0 + tid * per), i1 = min(g1, i0 + per);
    int64_t at;
    if (pick<WAVES>(sh, weigh, we, e, min_w, target, run, eq, i1 - i0, [&](int64_t i) {
            const uint32_t k = key_of(as_float<E>(row.x[i0 + i]));
            return row.tf && row.tf[i0 + i] >= a.T ? 0u : k;
        }, &at))
        put_winner(winners, n_win, b, i0 + at, row.tf ? (int)row.tf[i0 + at] : 0, a);
}

// Grid: one workgroup per row, top_k at most FEW_MAX: all three steps and the draw
// on the row's list, which as a rule holds little more than top_k entries.  Each
// entry is compared with all: how many come before it, the weight of those, and
// what is kept at lower indices.  Rows with more entries than a list takes (many
// scores of one bin) are read again instead.
constexpr int FEW_MAX = LIST / 4;
template <class E>
__global__ __launch_bounds__(LONG_THREADS) void k_sample_few(const E *__restrict__ scores,
                                                             const uint8_t *__restrict__ t_first,
                                                             const float *__restrict__ u, SampleArgs a, Work w,
                                                             int32_t *__restrict__ winners,
                                                             int32_t *__restrict__ n_win) {
    constexpr int WAVES = LONG_WAVES;
    __shared__ Shared<WAVES> sh;
    __shared__ uint64_t ent[LIST], wt[LIST], lead[LIST];  // entries, their weights, the weight before them
    const int64_t b = blockIdx.x;
    const int tid = threadIdx.x;
    const uint32_t n = w.count[b];
    const uint64_t mine = w.list[b * LIST + tid];  // (any bits behind n)
    const float draw = u[b];
    const RowStat st(w.part + b * w.splits, w.splits, a.temperature);
    if (st.n == 0) {  // nothing can win (uniform)
        if (tid < 4) winners[b * 4 + tid] = -1;
        if (tid == 0) n_win[b] = 0;
        return;
    }
    const Weigher weigh = weigher<WAVES>(sh, a, key_of(st.top));
    const uint64_t min_w = (uint64_t)ceil(ldexp((double)a.min_p, a.shift));
    const uint8_t *tf = t_first ? t_first + b * a.N : nullptr;
    __syncthreads();
    if (n <= LIST) {
        const uint32_t n8 = (n + 7) / 8 * 8;  // (entries 0 up to here: behind all others, of no weight)
        for (uint32_t i = tid; i < n8; i += LONG_THREADS) {
            const uint64_t x = i >= n ? 0 : i < LONG_THREADS ? mine : w.list[b * LIST + i];
            ent[i] = x;
            wt[i] = i < n ? weigh((uint32_t)(x >> 32)) : 0;
        }
        __syncthreads();
        uint64_t sum = 0;
        for (uint32_t i = tid; i < n; i += LONG_THREADS) {
            const uint64_t x = ent[i];
            uint64_t before = 0;
            uint32_t rank = 0;
            for (uint32_t j = 0; j < n8; j += 8) {
#pragma unroll
                for (int o = 0; o < 8; ++o) {
                    const bool first = ent[j + o] > x;
                    rank += first;
                    before += first ? wt[j + o] : 0;
                }
            }
            const bool in = rank < (uint32_t)a.top_k;
            lead[i] = in ? before : ~0ull;
            sum += in ? wt[i] : 0;
        }
        sum = block_sum<WAVES>(sh, sum);  // (after its barriers the weights have been read)
        const uint64_t want = a.top_p < 1.0f ? share(a.top_p, sum) : ~0ull;
        sum = 0;
        for (uint32_t i = tid; i < n; i += LONG_THREADS) {
            const uint64_t own = lead[i] < want && wt[i] >= min_w ? wt[i] : 0;
            wt[i] = own;
            sum += own;
        }
        const uint64_t target = target_of(draw, block_sum<WAVES>(sh, sum));
        for (uint32_t i = tid; i < n; i += LONG_THREADS) {
            if (wt[i] == 0) continue;
            const uint32_t x = (uint32_t)ent[i];
            uint64_t run = 0;
            for (uint32_t j = 0; j < n8; j += 8) {
#pragma unroll
                for (int o = 0; o < 8; ++o) run += (uint32_t)ent[j + o] > x ? wt[j + o] : 0;  // (a lower index)
            }
            if (target >= run && target < run + wt[i]) {
                const int64_t at = (uint32_t)~x;
                put_winner(winners, n_win, b, at, tf ? (int)tf[at] : 0, a);
            }
        }
        return;
    }
    const LongRow<E> row(scores, t_first, a, 1, b, 0);
    const Edge e = edge_of_count(sh, a, weigh, n, st.n,
                                 [&](const Edge &from, auto f, auto value) { row.each_from(from, f, value); });
    uint64_t we = weigh(e.edge), sum = 0, eqs = 0;
    we = we >= min_w && e.edge > 1 ? we : 0;
    row.all([&](float v, int64_t) {
        const uint32_t k = key_of(v);
        const uint64_t x = k > e.edge ? weigh(k) : 0;
        sum += x >= min_w ? x : 0;
        eqs += k == e.edge;
    });
    sum = block_sum<WAVES>(sh, sum);
    eqs = block_sum<WAVES>(sh, eqs);
    const uint64_t target = target_of(draw, sum + (eqs < e.equal ? eqs : e.equal) * we);
    const int64_t per = (a.N + LONG_THREADS - 1) / LONG_THREADS, i0 = min(a.N, tid * per), i1 = min(a.N, i0 + per);
    int64_t at;
    if (pick<WAVES>(sh, weigh, we, e, min_w, target, 0, 0, i1 - i0, [&](int64_t i) {
            const uint32_t k = key_of(as_float<E>(row.x[i0 + i]));
            return tf && tf[i0 + i] >= a.T ? 0u : k;
        }, &at))
        put_winner(winners, n_win, b, i0 + at, tf ? (int)tf[i0 + at] : 0, a);
}

constexpr int64_t SHORT_MAX = 16 * 64 * 16;  // keys of a row that the registers of a workgroup take

// Workgroups of a long row: one for each of 256 CUs in all (two of 1024 threads do
// not fit a CU's registers together: 32 rows of 131072 take 67 us with twice as
// many, 53 with these, 62 with half), and no less than 4096 scores each (8 rows of
// 50001 bfloat16 scores, top_k 50: 30.0 us from 2048 scores on, 28.6 from 4096; a row
// of 17000: 36.7 from 4096, 39.3 from 8192).
int splits_of(int B, int64_t N) {
    int64_t s = 256 / B;
    s = s < N / 4096 ? s : N / 4096;
    return (int)(s < 1 ? 1 : s > SPLITS ? SPLITS : s);
}

size_t carve(void *ws, int B, int64_t N, Work *w) {
    spk::Carver c(ws);
    w->splits = splits_of(B, N);
    w->hist = c.take<uint64_t>((size_t)B * BINS);
    w->list = c.take<uint64_t>((size_t)B * LIST);
    w->count = c.take<uint32_t>(B);
    w->part = c.take<RowPart>((size_t)B * w->splits);
    w->sums = c.take<RowSums>((size_t)B * w->splits * LONG_WAVES);
    w->edge = c.take<RowEdge>(B);
    return spk::align_up(c.off, 256);
}

template <class E>
void launch(const void *scores, const uint8_t *t_first, const float *u, int B, const SampleArgs &a, int32_t *winners,
            int32_t *n_winners, void *ws, hipStream_t st) {
    const E *x = static_cast<const E *>(scores);
    const dim3 rows((unsigned)B), threads(LONG_THREADS);
    // As few waves as hold the row, so that more workgroups share a CU and one's steps
    // fill the other's waits: 1000 rows of 2000 take 17.7 us with two waves each, 21.7
    // with four; of 8000 45 us with eight, 95 with sixteen, 121 by the launches below
    // (of 16000: 120 with sixteen, 148 below; 16 such rows 37.3 and 38.6).
#define SPK_SHORT(WAVES)                                                                                        \
    if (a.N <= WAVES * 64 * 16) {                                                                               \
        hipLaunchKernelGGL((k_sample_short<E, WAVES>), rows, dim3(WAVES * 64), 0, st, x, t_first, u, a, winners, \
                           n_winners);                                                                          \
        return;                                                                                                 \
    }
    SPK_SHORT(2)
    SPK_SHORT(4)
    SPK_SHORT(8)
    SPK_SHORT(16)
#undef SPK_SHORT
    Work w;
    carve(ws, B, a.N, &w);
    const dim3 grid((unsigned)w.splits, (unsigned)B);
    hipLaunchKernelGGL(k_sample_top<E>, grid, threads, 0, st, x, t_first, a, w);
    const bool one = a.temperature == 0.0f || a.top_k == 1, by_count = !one && a.top_k > 0 && a.top_k < a.N;
    if (by_count) {
        hipLaunchKernelGGL((k_sample_hist<E, true>), grid, threads, 0, st, x, t_first, a, w);
        hipLaunchKernelGGL((k_sample_list<E, true>), grid, threads, 0, st, x, t_first, a, w);
        if (a.top_k <= FEW_MAX) {
            hipLaunchKernelGGL(k_sample_few<E>, rows, threads, 0, st, x, t_first, u, a, w, winners, n_winners);
            return;
        }
        hipLaunchKernelGGL((k_sample_sums<E, 2>), grid, threads, 0, st, x, t_first, a, w);
    } else if (!one && a.top_p < 1.0f) {
        hipLaunchKernelGGL((k_sample_hist<E, false>), grid, threads, 0, st, x, t_first, a, w);
        hipLaunchKernelGGL((k_sample_list<E, false>), grid, threads, 0, st, x, t_first, a, w);
        hipLaunchKernelGGL((k_sample_sums<E, 1>), grid, threads, 0, st, x, t_first, a, w);
    } else {
        hipLaunchKernelGGL((k_sample_sums<E, 0>), grid, threads, 0, st, x, t_first, a, w);
    }
    hipLaunchKernelGGL(k_sample_pick<E>, rows, threads, 0, st, x, t_first, u, a, w, winners, n_winners);
}

int check(int dtype, int B, int C, int H, int W, const char *name) {
    SPK_REQUIRE(dtype == SPK_F32 || dtype == SPK_BF16, SPK_E_ARG, "%s: dtype %d is neither SPK_F32 nor SPK_BF16", name,
                dtype);
    SPK_REQUIRE(B >= 0 && C >= 1 && H >= 1 && W >= 1, SPK_E_SHAPE, "%s: bad sizes", name);
    SPK_REQUIRE((int64_t)C * H <= (1 << 24) && (int64_t)C * H * W <= (1 << 24), SPK_E_RANGE, "%s: C*H*W above 2^24",
                name);
    // (a workgroup an image, of up to 1024 threads; long rows have a grid dimension for the images)
    SPK_REQUIRE(B <= (1 << 21) && ((int64_t)C * H * W <= SHORT_MAX || B <= 65535), SPK_E_RANGE,
                "%s: B=%d above 2^21, or above 65535 with C*H*W above 16384", name, B);
    return SPK_OK;
}

}  // namespace

extern "C" size_t spk_sample_winners_workspace_size(int dtype, int B, int C, int H, int W) {
    if (check(dtype, B, C, H, W, "") != SPK_OK || B == 0) return 0;
    const int64_t N = (int64_t)C * H * W;
    Work w;
    return N > SHORT_MAX ? carve(nullptr, B, N, &w) : 0;
}

extern "C" int spk_sample_winners(const void *scores, int dtype, const uint8_t *t_first, const float *u, int B, int T,
                                  int C, int H, int W, float temperature, int top_k, float top_p, float min_p,
                                  int32_t *winners, int32_t *n_winners, void *workspace, size_t ws_bytes,
                                  void *stream) {
    const char *name = "spk_sample_winners";
    if (int rc = check(dtype, B, C, H, W, name)) return rc;
    SPK_REQUIRE(T >= 1, SPK_E_SHAPE, "%s: bad sizes", name);
    SPK_REQUIRE(T <= 255, SPK_E_RANGE, "%s: T=%d > 255", name, T);
    SPK_REQUIRE(temperature >= 0.0f && std::isfinite(temperature), SPK_E_ARG, "%s: temperature must be finite and >= 0",
                name);
    SPK_REQUIRE(top_k >= 0, SPK_E_ARG, "%s: top_k=%d < 0", name, top_k);
    SPK_REQUIRE(top_p > 0.0f && top_p <= 1.0f, SPK_E_ARG, "%s: top_p must be in (0, 1]", name);
    SPK_REQUIRE(min_p >= 0.0f && min_p <= 1.0f, SPK_E_ARG, "%s: min_p must be in [0, 1]", name);
    if (B == 0) return spk::ok();
    SPK_REQUIRE(scores && u && winners && n_winners, SPK_E_ARG, "%s: scores, u, winners and n_winners are required",
                name);
    const size_t need = spk_sample_winners_workspace_size(dtype, B, C, H, W);
    SPK_REQUIRE(need == 0 || (workspace && ws_bytes >= need), SPK_E_WORKSPACE, "%s: workspace of %zu bytes, %zu needed",
                name, workspace ? ws_bytes : (size_t)0, need);
    SPK_REQUIRE(need == 0 || (reinterpret_cast<uintptr_t>(workspace) & 15) == 0, SPK_E_ARG,
                "%s: the workspace must be 16-byte aligned", name);
    SampleArgs a;
    a.N = (int64_t)C * H * W;
    a.T = T;
    a.HW = H * W;
    a.W = W;
    a.top_k = top_k;
    a.temperature = temperature;
    a.top_p = top_p;
    a.min_p = min_p;
    int lg = 0;
    while ((1ll << lg) < a.N) ++lg;
    a.shift = std::min(51, 62 - lg);
    hipStream_t st = spk::as_stream(stream);
    if (dtype == SPK_F32) launch<float>(scores, t_first, u, B, a, winners, n_winners, workspace, st);
    else launch<uint16_t>(scores, t_first, u, B, a, winners, n_winners, workspace, st);
    return spk::check_launch(name);
}
