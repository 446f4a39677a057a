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
// Rows of up to 16 keys a thread stay in registers.  Longer ones are read again
// for each step (largest score; histogram; the boundary's own bin into LDS; sums
// by index): a step is bound by reading the row, and beside it the weights cost
// some 20 double-precision instructions a score.
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

constexpr int POW = 128;    // entries of the table of 2^(j / POW)
constexpr int BINS = 2048;  // bins of a row's first histogram
constexpr int LIST = 4096;  // keys of one bin that LDS takes

// Weights of a row: floor(2^shift exp((score - largest) / temperature)).  With
// y = shift + (score - largest) log2(e) / temperature = n + j / POW + r, it is
// 2^n 2^(j / POW) 2^r with 2^r from its series: the last term left out,
// (r ln 2)^6 / 720, is below 4e-17.  The largest itself (also +inf) weighs 2^shift.
struct Weigher {
    double top, per, shift_d;
    uint32_t ktop;
    int shift;
    const double *pow;
    __device__ __forceinline__ uint64_t operator()(uint32_t k) const {
        if (k == ktop) return 1ull << shift;
        const double y = fmax(fma((double)value_of(k) - top, per, shift_d), -1.0);
        const double n = floor(y), f = y - n;
        const int j = (int)(f * POW);
        const double t = (f - j * (1.0 / POW)) * 0.69314718055994530942;
        double p = fma(t, 1.0 / 120, 1.0 / 24);
        p = fma(t, p, 1.0 / 6);
        p = fma(t, p, 0.5);
        p = fma(t, p, 1.0);
        p = fma(t, p, 1.0);
        const uint64_t bits = __double_as_longlong(pow[j & (POW - 1)] * p);  // in [1, 2]
        // the significand as an integer times 2^(n - 52), and 2^n a bit on where rounding reached 2
        const int e = (int)n + (int)(bits >> 52) - 1023 - 52;
        const uint64_t sig = (bits & 0xFFFFFFFFFFFFFull) | 0x10000000000000ull;
        const uint64_t w = e >= 0 ? sig << e : sig >> -e;
        return y >= 0.0 ? w : 0ull;
    }
};

// LDS of a row's workgroup of WAVES waves.
template <int WAVES>
struct Shared {
    uint64_t hist[BINS];
    double pow[POW];
    uint64_t part[WAVES], part2[WAVES];
    uint64_t above;
    uint32_t bin, n_list;
    uint32_t list[LIST];
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

// The first of n bins (from bin 0) at which the running total reaches `want`,
// the last one if it never does; *above gets the total of the bins before it.
template <int WAVES>
__device__ __forceinline__ uint32_t find_bin(Shared<WAVES> &sh, int n, uint64_t want, uint64_t *above) {
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x, per = n / 64;
        uint64_t sum = 0;
        for (int j = 0; j < per; ++j) sum += sh.hist[lane * per + j];
        const uint64_t incl = wave_scan_u64(sum, lane);
        const uint64_t hit = __ballot(incl >= want);
        const int src = hit ? __ffsll((unsigned long long)hit) - 1 : 63;
        if (lane == src) {
            uint64_t run = incl - sum;
            int j = 0;
            for (; j < per - 1 && run + sh.hist[lane * per + j] < want; ++j) run += sh.hist[lane * per + j];
            sh.bin = (uint32_t)(lane * per + j);
            sh.above = run;
        }
    }
    __syncthreads();
    *above = sh.above;
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
        const uint32_t bin = find_bin<WAVES>(sh, 256, want - above, &over);
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
    if (threadIdx.x < POW) sh.pow[threadIdx.x] = exp2(threadIdx.x * (1.0 / POW));
    Weigher w;
    w.ktop = ktop;
    w.top = (double)value_of(ktop);
    w.per = a.temperature > 0.0f ? 1.4426950408889634074 / (double)a.temperature : 0.0;
    w.shift = a.shift;
    w.shift_d = (double)a.shift;
    w.pow = sh.pow;
    return w;
}

// The draw among `n` keys of a thread that follow each other in index (0 =
// cannot win): keys above the edge and the first `equal` equal to it, of weight
// min_w at least.  key_at(i) gives the thread's i-th key, weight_at(i, key) its
// weight.  `run`, `eq`: kept weight and equal keys before the workgroup's first.
// Returns whether this thread holds the winner, and its number.
template <int WAVES, class KeyAt, class WeightAt>
__device__ __forceinline__ bool pick(Shared<WAVES> &sh, uint64_t we, const Edge &e, uint64_t min_w, uint64_t target,
                                     uint64_t run, uint64_t eq, int64_t n, KeyAt key_at, WeightAt weight_at,
                                     int64_t *at) {
    constexpr int AHEAD = 8;  // keys read at a time
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    uint64_t sum = 0, eqs = 0;
    for (int64_t i = 0; i < n; i += AHEAD) {
        uint32_t k[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) k[j] = key_at(min(i + j, n - 1));
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            if (i + j >= n) continue;
            const uint64_t w = k[j] > e.edge ? weight_at(i + j, k[j]) : 0;
            sum += w >= min_w ? w : 0;
            eqs += k[j] == e.edge;
        }
    }
    const uint64_t si = wave_scan_u64(sum, lane), ei = wave_scan_u64(eqs, lane);
    __syncthreads();
    if (lane == 63) {
        sh.part[wv] = si;
        sh.part2[wv] = ei;
    }
    __syncthreads();
    for (int q = 0; q < wv; ++q) {
        run += sh.part[q];
        eq += sh.part2[q];
    }
    run += si - sum;
    eq += ei - eqs;
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
            w = weight_at(i, k);
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

// Grid: one workgroup per image, whose row of at most 16 keys a thread stays in
// registers; a thread's keys follow each other in index.
template <class E, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void k_sample_short(const E *__restrict__ scores,
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
    uint64_t top = 0, cnt = 0;
#pragma unroll
    for (int j = 0; j < KEYS; ++j) {
        key[j] = j < per && i0 + j < N ? key[j] : 0u;
        top = key[j] > top ? key[j] : top;
        cnt += key[j] != 0;
    }
    top = spk::wave_max_u64(top);
    if ((tid & 63) == 0) sh.part2[tid >> 6] = top;
    const uint64_t total = block_sum<WAVES>(sh, cnt);
#pragma unroll
    for (int q = 0; q < WAVES; ++q) top = sh.part2[q] > top ? sh.part2[q] : top;
    if (top == 0) {  // nothing can win (uniform)
        if (tid < 4) winners[b * 4 + tid] = -1;
        if (tid == 0) n_win[b] = 0;
        return;
    }
    const Weigher weigh = weigher<WAVES>(sh, a, (uint32_t)top);
    __syncthreads();
    Edge e;
    uint64_t above;
    const uint64_t top_k = a.temperature > 0.0f ? (uint64_t)a.top_k : 1ull;
    if (top_k == 1) {
        e.edge = (uint32_t)top;
        e.equal = 1;
    } else if (top_k > 0 && top_k < total) {
        e.edge = descend<WAVES>(sh, top_k, [&](auto f) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
                if (key[j]) f(key[j], [] { return (uint64_t)1; });
        }, &above);
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
        const uint32_t k = descend<WAVES>(sh, want, [&](auto f) {
#pragma unroll
            for (int j = 0; j < KEYS; ++j)
                if (w[j]) f(key[j], [&] { return w[j]; });
        }, &above);
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
    sum = block_sum<WAVES>(sh, sum);
    eqs = block_sum<WAVES>(sh, eqs);
    const uint64_t target = target_of(u[b], sum + (eqs < e.equal ? eqs : e.equal) * we);
    int64_t at;
    if (pick<WAVES>(sh, we, e, min_w, target, 0, 0, per, [&](int64_t i) {
            uint32_t k = 0;
#pragma unroll
            for (int j = 0; j < KEYS; ++j) k = j == i ? key[j] : k;
            return k;
        }, [&](int64_t i, uint32_t) {
            uint64_t x = 0;
#pragma unroll
            for (int j = 0; j < KEYS; ++j) x = j == i ? w[j] : x;
            return x;
        }, &at))
        put_winner(winners, n_win, b, i0 + at, tf ? (int)tf[i0 + at] : 0, a);
}

constexpr int LONG_WAVES = 16, LONG_THREADS = LONG_WAVES * 64;

// Calls f(key, index) for the keys i0 <= index < i1 of a row, by `threads`
// threads of which this is number `t`: vectors of 16 bytes, four in flight a
// thread, and the ends that no whole vector covers one by one.  A key that
// cannot win is 0.
template <class E, class F>
__device__ __forceinline__ void for_row(const E *x, const uint8_t *tf, int T, int64_t i0, int64_t i1, int t, int threads,
                                        F f) {
    constexpr int V = 16 / sizeof(E), UNR = 4;
    auto one = [&](int64_t i) {
        f(tf && tf[i] >= T ? 0u : key_of(as_float<E>(x[i])), i);
    };
    const int64_t skip = (V - (int64_t)((reinterpret_cast<uintptr_t>(x + i0) / sizeof(E)) % V)) % V;
    const int64_t v0 = min(i1, i0 + skip), nv = (i1 - v0) / V;
    struct alignas(16) Vec {
        E e[V];
    };
    const Vec *xv = reinterpret_cast<const Vec *>(x + v0);
    for (int64_t j = t; j < nv; j += (int64_t)threads * UNR) {
        Vec r[UNR];
#pragma unroll
        for (int q = 0; q < UNR; ++q) r[q] = xv[min(j + (int64_t)q * threads, nv - 1)];
        if (tf) {
            uint8_t tt[UNR][V];
#pragma unroll
            for (int q = 0; q < UNR; ++q)
#pragma unroll
                for (int c = 0; c < V; ++c) tt[q][c] = tf[v0 + min(j + (int64_t)q * threads, nv - 1) * V + c];
#pragma unroll
            for (int q = 0; q < UNR; ++q)
                if (j + (int64_t)q * threads < nv)
#pragma unroll
                    for (int c = 0; c < V; ++c)
                        f(tt[q][c] < T ? key_of(as_float<E>(r[q].e[c])) : 0u, v0 + (j + (int64_t)q * threads) * V + c);
        } else {
#pragma unroll
            for (int q = 0; q < UNR; ++q)
                if (j + (int64_t)q * threads < nv)
#pragma unroll
                    for (int c = 0; c < V; ++c)
                        f(key_of(as_float<E>(r[q].e[c])), v0 + (j + (int64_t)q * threads) * V + c);
        }
    }
    const int64_t head = v0 - i0, tail = i1 - v0 - nv * V;  // below V each
    if (t < head) one(i0 + t);
    else if (t - head < tail) one(i1 - tail + (t - head));
}

// Grid: one workgroup per image of any size.  A boundary is looked for in a
// histogram of BINS equal steps of the score below the largest (1/64 of the
// temperature each, the rest in the last), then among the keys of its bin, in
// LDS where they fit; else by reading the row again for every digit.
template <class E>
__global__ __launch_bounds__(LONG_THREADS) void k_sample_long(const E *__restrict__ scores,
                                                              const uint8_t *__restrict__ t_first,
                                                              const float *__restrict__ u, SampleArgs a,
                                                              int32_t *__restrict__ winners,
                                                              int32_t *__restrict__ n_win) {
    constexpr int WAVES = LONG_WAVES;
    __shared__ Shared<WAVES> sh;
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t b = blockIdx.x, N = a.N;
    const E *x = scores + b * N;
    const uint8_t *tf = t_first ? t_first + b * N : nullptr;
    auto each = [&](auto f) { for_row<E>(x, tf, a.T, 0, N, tid, LONG_THREADS, f); };
    uint32_t mx = 0, c32 = 0;
    each([&](uint32_t k, int64_t) {
        mx = k > mx ? k : mx;
        c32 += k != 0;
    });
    uint64_t top = spk::wave_max_u64(mx);
    if (lane == 0) sh.part2[wv] = top;
    const uint64_t total = block_sum<WAVES>(sh, c32);
#pragma unroll
    for (int q = 0; q < WAVES; ++q) top = sh.part2[q] > top ? sh.part2[q] : top;
    if (top == 0) {  // nothing can win (uniform)
        if (tid < 4) winners[b * 4 + tid] = -1;
        if (tid == 0) n_win[b] = 0;
        return;
    }
    const Weigher weigh = weigher<WAVES>(sh, a, (uint32_t)top);
    const float ftop = value_of((uint32_t)top), steps = a.temperature > 0.0f ? 64.0f / a.temperature : 1.0f;
    auto bin_of = [&](uint32_t k) -> int {  // does not fall as the score falls
        return k == (uint32_t)top ? 0 : (int)fminf((ftop - value_of(k)) * steps, (float)(BINS - 1));
    };
    Edge e;
    // moves the boundary to where the running total of value() reaches `want`; returns the new
    // key and, in *above, the total of the larger ones
    auto narrow = [&](uint64_t want, auto value, uint64_t *above) -> uint32_t {
        const uint32_t from = e.edge;
        for (int i = tid; i < BINS; i += LONG_THREADS) sh.hist[i] = 0;
        if (tid == 0) sh.n_list = 0;
        __syncthreads();
        each([&](uint32_t k, int64_t) {
            if (k >= from) {
                const uint64_t v = value(k);
                if (v) atomicAdd((unsigned long long *)&sh.hist[bin_of(k)], (unsigned long long)v);
            }
        });
        uint64_t over, in;
        const int bin = (int)find_bin<WAVES>(sh, BINS, want, &over);
        each([&](uint32_t k, int64_t) {
            if (k >= from && bin_of(k) == bin) {
                const uint32_t at = atomicAdd(&sh.n_list, 1u);
                if (at < LIST) sh.list[at] = k;
            }
        });
        __syncthreads();
        const uint32_t n = sh.n_list;
        uint32_t key;
        if (n <= LIST)
            key = descend<WAVES>(sh, want - over, [&](auto f) {
                for (uint32_t i = tid; i < n; i += LONG_THREADS) {
                    const uint32_t k = sh.list[i];
                    f(k, [&] { return value(k); });
                }
            }, &in);
        else
            key = descend<WAVES>(sh, want - over, [&](auto f) {
                each([&](uint32_t k, int64_t) {
                    if (k >= from && bin_of(k) == bin) f(k, [&] { return value(k); });
                });
            }, &in);
        *above = over + in;
        return key;
    };
    uint64_t above;
    const uint64_t top_k = a.temperature > 0.0f ? (uint64_t)a.top_k : 1ull;
    if (top_k == 1) {
        e.edge = (uint32_t)top;
        e.equal = 1;
    } else if (top_k > 0 && top_k < total) {
        const uint32_t k = narrow(top_k, [](uint32_t) -> uint64_t { return 1; }, &above);
        e.edge = k;
        e.equal = top_k - above;
    }
    __syncthreads();
    if (a.top_p < 1.0f && top_k != 1) {
        uint64_t sum = 0;
        each([&](uint32_t k, int64_t) {
            if (k > e.edge || (k == e.edge && e.equal == ~0ull)) sum += weigh(k);
        });
        sum = block_sum<WAVES>(sh, sum);
        if (e.equal != ~0ull) sum += e.equal * weigh(e.edge);
        const uint64_t want = share(a.top_p, sum);
        const uint32_t k = narrow(want, weigh, &above);
        e.by_weight(k, want, above, weigh(k));
    }
    const uint64_t min_w = (uint64_t)ceil(ldexp((double)a.min_p, a.shift));
    uint64_t we = weigh(e.edge);
    we = we >= min_w ? we : 0;
    // sums of the waves' segments of the row, and the segment of the draw
    const int64_t seg = ((N + WAVES - 1) / WAVES + 63) / 64 * 64;
    uint64_t sum = 0, eqs = 0;
    for_row<E>(x, tf, a.T, min(N, wv * seg), min(N, (wv + 1) * seg), lane, 64, [&](uint32_t k, int64_t) {
        const uint64_t w = k > e.edge ? weigh(k) : 0;
        sum += w >= min_w ? w : 0;
        eqs += k == e.edge;
    });
    sum = wave_sum_u64(sum);
    eqs = wave_sum_u64(eqs);
    __syncthreads();
    if (lane == 0) {
        sh.part[wv] = sum;
        sh.part2[wv] = eqs;
    }
    __syncthreads();
    uint64_t left = e.equal, all = 0;
    for (int q = 0; q < WAVES; ++q) {
        const uint64_t m = sh.part2[q] < left ? sh.part2[q] : left;
        left -= m;
        all += sh.part[q] + m * we;
    }
    const uint64_t target = target_of(u[b], all);
    uint64_t run = 0, eq = 0;
    int at_seg = 0;
    for (int q = 0; q < WAVES; ++q) {
        const uint64_t used = eq < e.equal ? eq : e.equal;
        const uint64_t m = sh.part2[q] < e.equal - used ? sh.part2[q] : e.equal - used;
        if (target < run + used * we + sh.part[q] + m * we) {
            at_seg = q;
            break;
        }
        run += sh.part[q];
        eq += sh.part2[q];
    }
    const int64_t g0 = min(N, at_seg * seg), g1 = min(N, g0 + seg), per = (g1 - g0 + LONG_THREADS - 1) / LONG_THREADS;
    const int64_t i0 = min(g1, g0 + tid * per), i1 = min(g1, i0 + per);
    int64_t at;
    if (pick<WAVES>(sh, we, e, min_w, target, run, eq, i1 - i0, [&](int64_t i) {
            const uint32_t k = key_of(as_float<E>(x[i0 + i]));
            return tf && tf[i0 + i] >= a.T ? 0u : k;
        }, [&](int64_t, uint32_t k) { return weigh(k); }, &at))
        put_winner(winners, n_win, b, i0 + at, tf ? (int)tf[i0 + at] : 0, a);
}

template <class E>
void launch(const void *scores, const uint8_t *t_first, const float *u, int B, const SampleArgs &a, int32_t *winners,
            int32_t *n_winners, hipStream_t st) {
    const E *x = static_cast<const E *>(scores);
    const dim3 grid((unsigned)B);
    if (a.N <= 4 * 64 * 16)
        hipLaunchKernelGGL((k_sample_short<E, 4>), grid, dim3(256), 0, st, x, t_first, u, a, winners, n_winners);
    else if (a.N <= 16 * 64 * 16)
        hipLaunchKernelGGL((k_sample_short<E, 16>), grid, dim3(1024), 0, st, x, t_first, u, a, winners, n_winners);
    else
        hipLaunchKernelGGL(k_sample_long<E>, grid, dim3(LONG_THREADS), 0, st, x, t_first, u, a, winners, n_winners);
}

}  // namespace

extern "C" size_t spk_sample_winners_workspace_size(int dtype, int B, int C, int H, int W) {
    (void)dtype, (void)B, (void)C, (void)H, (void)W;
    return 0;
}

extern "C" int spk_sample_winners(const void *scores, int dtype, const uint8_t *t_first, const float *u, int B, int T,
                                  int C, int H, int W, float temperature, int top_k, float top_p, float min_p,
                                  int32_t *winners, int32_t *n_winners, void *workspace, size_t ws_bytes,
                                  void *stream) {
    const char *name = "spk_sample_winners";
    SPK_REQUIRE(dtype == SPK_F32 || dtype == SPK_BF16, SPK_E_ARG, "%s: dtype %d is neither SPK_F32 nor SPK_BF16", name,
                dtype);
    SPK_REQUIRE(B >= 0 && C >= 1 && H >= 1 && W >= 1 && T >= 1, SPK_E_SHAPE, "%s: bad sizes", name);
    SPK_REQUIRE(T <= 255, SPK_E_RANGE, "%s: T=%d > 255", name, T);
    SPK_REQUIRE((int64_t)C * H <= (1 << 24) && (int64_t)C * H * W <= (1 << 24), SPK_E_RANGE, "%s: C*H*W above 2^24",
                name);
    SPK_REQUIRE(B <= (1 << 21), SPK_E_RANGE, "%s: B=%d > 2^21", name, B);
    SPK_REQUIRE(temperature >= 0.0f && std::isfinite(temperature), SPK_E_ARG, "%s: temperature must be finite and >= 0",
                name);
    SPK_REQUIRE(top_k >= 0, SPK_E_ARG, "%s: top_k=%d < 0", name, top_k);
    SPK_REQUIRE(top_p > 0.0f && top_p <= 1.0f, SPK_E_ARG, "%s: top_p must be in (0, 1]", name);
    SPK_REQUIRE(min_p >= 0.0f && min_p <= 1.0f, SPK_E_ARG, "%s: min_p must be in [0, 1]", name);
    if (B == 0) return spk::ok();
    SPK_REQUIRE(scores && u && winners && n_winners, SPK_E_ARG, "%s: scores, u, winners and n_winners are required",
                name);
    (void)workspace, (void)ws_bytes;
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
    a.shift = 62 - lg;
    hipStream_t st = spk::as_stream(stream);
    if (dtype == SPK_F32) launch<float>(scores, t_first, u, B, a, winners, n_winners, st);
    else launch<uint16_t>(scores, t_first, u, B, a, winners, n_winners, st);
    return spk::check_launch(name);
}
