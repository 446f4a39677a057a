// One winner per image drawn from its neurons' scores (gfx950).
//
// The order of the definition is that of the pairs (score from largest, index
// from smallest).  What steps 1 and 2 keep is a prefix of that order, so it is
// described by a boundary: every score above it, and the first `equal` indices
// of the scores equal to it.  A boundary is found on order-preserving 32-bit
// keys, a digit at a time from the highest, by a histogram of the keys that
// share the digits found so far: of counts for top_k, of weights for top_p.
// Weights are 64-bit fixed-point numbers, so that a histogram built by atomics
// does not depend on their order.
#include <cmath>

#include "common.hpp"
#include "libspyke_readout.h"

namespace {

constexpr int WAVES = 16;
constexpr int THREADS = WAVES * 64;

struct SampleArgs {
    int64_t N;  // neurons of an image
    int B, T, HW, W, top_k, shift;  // shift: fraction bits of a weight
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

struct Row {
    double inv_t;   // 1 / temperature
    double top;     // largest score
    uint32_t ktop;
    int shift;
    // exp((score - largest) / temperature); the largest itself (also +inf) weighs 1
    __device__ __forceinline__ double ratio(uint32_t k) const {
        return k == ktop ? 1.0 : exp(((double)value_of(k) - top) * inv_t);
    }
    __device__ __forceinline__ uint64_t weight(uint32_t k) const { return (uint64_t)ldexp(ratio(k), shift); }
};

// Largest position p of a boundary search over 256 bins from the highest: the
// bin in which the running total first reaches `want`; *above gets the total
// of the bins over it.  hist is in LDS; called by the first wave.
__device__ __forceinline__ int find_bin(const uint64_t *hist, uint64_t want, uint64_t *above) {
    const int lane = threadIdx.x & 63;
    uint64_t own[4], sum = 0;  // lane's bins 255 - 4*lane - j, from the highest
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += own[j] = hist[255 - 4 * lane - j];
    uint64_t incl = sum;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const uint64_t o = __shfl_up(incl, s, 64);
        if (lane >= s) incl += o;
    }
    const uint64_t hit = __ballot(incl >= want);
    const int src = hit ? __ffsll((unsigned long long)hit) - 1 : 63;
    uint64_t run = incl - sum;
    int bin = 255 - 4 * lane - 3;
    bool found = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (!found && run + own[j] >= want) {
            bin = 255 - 4 * lane - j;
            found = true;
        }
        if (!found) run += own[j];
    }
    if (!found) run -= own[3];  // (the last bin stands in when the total stays below `want`)
    *above = __shfl(run, src, 64);
    return __shfl(bin, src, 64);
}

// Grid: one workgroup per image.
template <class E>
__global__ __launch_bounds__(THREADS) void k_sample_row(const E *__restrict__ scores,
                                                        const uint8_t *__restrict__ t_first,
                                                        const float *__restrict__ u, SampleArgs a,
                                                        int32_t *__restrict__ winners, int32_t *__restrict__ n_win) {
    __shared__ uint64_t hist[256];
    __shared__ uint64_t part[WAVES], parteq[WAVES];
    __shared__ uint64_t s_above;
    __shared__ uint32_t s_bin;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int64_t b = blockIdx.x, N = a.N;
    const E *x = scores + b * N;
    const uint8_t *tf = t_first ? t_first + b * N : nullptr;
    auto key_at = [&](int64_t i) -> uint32_t {
        if (i >= N || (tf && tf[i] >= a.T)) return 0u;
        return key_of(as_float<E>(x[i]));
    };
    // largest key and the number of eligible neurons
    uint32_t top = 0;
    uint64_t cnt = 0;
    for (int64_t i = tid; i < N; i += THREADS) {
        const uint32_t k = key_at(i);
        top = k > top ? k : top;
        cnt += k != 0;
    }
    const uint64_t tw = spk::wave_max_u64(top);
    cnt = wave_sum_u64(cnt);
    if (lane == 0) {
        part[wv] = tw;
        parteq[wv] = cnt;
    }
    __syncthreads();
    uint64_t ktop = 0, total = 0;
    for (int q = 0; q < WAVES; ++q) {
        ktop = part[q] > ktop ? part[q] : ktop;
        total += parteq[q];
    }
    __syncthreads();
    if (ktop == 0) {  // nothing can win (uniform)
        if (tid < 4) winners[b * 4 + tid] = -1;
        if (tid == 0) n_win[b] = 0;
        return;
    }
    Row row;
    row.ktop = (uint32_t)ktop;
    row.top = (double)value_of((uint32_t)ktop);
    row.inv_t = a.temperature > 0.0f ? 1.0 / (double)a.temperature : 0.0;
    row.shift = a.shift;
    // the boundary: keys above `edge` stay, and the first `equal` of those equal to it
    uint32_t edge = 1;
    uint64_t equal = ~0ull;
    const uint64_t top_k = a.temperature > 0.0f ? (uint64_t)a.top_k : 1ull;

    // boundary at which the running total of value(k) from the largest key reaches `want`,
    // among the keys that the present boundary keeps; the digits of `edge` are found in turn
    auto descend = [&](uint64_t want, auto value, uint64_t *above_edge) -> uint32_t {
        uint32_t prefix = 0;
        uint64_t above = 0;
        for (int sh = 24; sh >= 0; sh -= 8) {
            for (int i = tid; i < 256; i += THREADS) hist[i] = 0;
            __syncthreads();
            for (int64_t i = tid; i < N; i += THREADS) {
                const uint32_t k = key_at(i);
                if (k >= edge && (sh == 24 || (k >> (sh + 8)) == prefix)) {
                    const uint64_t v = value(k);
                    if (v) atomicAdd((unsigned long long *)&hist[(k >> sh) & 255], (unsigned long long)v);
                }
            }
            __syncthreads();
            if (wv == 0) {
                uint64_t over;
                const int bin = find_bin(hist, want - above, &over);
                if (lane == 0) {
                    s_bin = (uint32_t)bin;
                    s_above = over;
                }
            }
            __syncthreads();
            prefix = (prefix << 8) | s_bin;
            above += s_above;
            __syncthreads();
        }
        *above_edge = above;
        return prefix;
    };
    uint64_t above;
    if (top_k > 0 && top_k < total) {
        const uint32_t e = descend(top_k, [](uint32_t) -> uint64_t { return 1; }, &above);
        edge = e;
        equal = top_k - above;
    }
    if (a.top_p < 1.0f && a.temperature > 0.0f) {
        // the sum of what step 1 keeps: the keys above the edge and `equal` times the edge's weight
        uint64_t sum = 0;
        for (int64_t i = tid; i < N; i += THREADS) {
            const uint32_t k = key_at(i);
            if (k > edge || (k == edge && equal == ~0ull)) sum += row.weight(k);
        }
        sum = wave_sum_u64(sum);
        if (lane == 0) part[wv] = sum;
        __syncthreads();
        sum = 0;
        for (int q = 0; q < WAVES; ++q) sum += part[q];
        __syncthreads();
        const uint64_t we = row.weight(edge);
        if (equal != ~0ull) sum += equal * we;
        uint64_t want = (uint64_t)ceil((double)a.top_p * (double)sum);
        want = want < 1 ? 1 : (want > sum ? sum : want);
        const uint32_t e = descend(want, [&](uint32_t k) { return row.weight(k); }, &above);
        // (the edge of step 1 takes part with all its equals: one that step 1 cut has its own limit)
        const uint64_t w2 = row.weight(e);
        const uint64_t m = w2 ? (want - above + w2 - 1) / w2 : 1;
        equal = e == edge ? (m < equal ? m : equal) : m;
        edge = e;
    }
    // step 3 and the draw: each wave sums its segment of the indices
    const int64_t seg = (N + WAVES * 64 - 1) / (WAVES * 64) * 64;
    const int64_t i0 = wv * seg, i1 = min(N, i0 + seg);
    uint64_t sum = 0, eq = 0;
    for (int64_t i = i0 + lane; i < i1; i += 64) {
        const uint32_t k = key_at(i);
        if (k > edge) {
            const double r = row.ratio(k);
            if (r >= (double)a.min_p) sum += (uint64_t)ldexp(r, a.shift);
        }
        eq += k == edge;
    }
    sum = wave_sum_u64(sum);
    eq = wave_sum_u64(eq);
    if (lane == 0) {
        part[wv] = sum;
        parteq[wv] = eq;
    }
    __syncthreads();
    // the edge's weight, 0 where min_p drops it
    const double re = row.ratio(edge);
    const uint64_t we = re >= (double)a.min_p ? (uint64_t)ldexp(re, a.shift) : 0;
    uint64_t left = equal, all = 0;
    for (int q = 0; q < WAVES; ++q) {
        const uint64_t e = parteq[q] < left ? parteq[q] : left;
        left -= e;
        all += part[q] + e * we;
    }
    const float uf = u[b];
    const double ud = uf > 0.0f ? fmin((double)uf, 1.0) : 0.0;
    uint64_t target = (uint64_t)(ud * (double)all);
    target = target < all ? target : all - 1;  // all >= the largest's weight
    uint64_t run = 0;
    left = equal;
    int at = -1;
    for (int q = 0; q < WAVES; ++q) {  // the segment that holds the target
        const uint64_t e = parteq[q] < left ? parteq[q] : left;
        const uint64_t s = part[q] + e * we;
        if (at < 0) {
            if (run + s > target) at = q;
            else {
                run += s;
                left -= e;
            }
        }
    }
    if (wv != at) return;
    for (int64_t i = i0; i < i1; i += 64) {
        const uint32_t k = key_at(i + lane < i1 ? i + lane : N);
        const uint64_t eqm = __ballot(k == edge);
        const uint64_t before = __popcll(eqm & ((1ull << lane) - 1ull));
        uint64_t w = 0;
        if (k > edge) {
            const double r = row.ratio(k);
            if (r >= (double)a.min_p) w = (uint64_t)ldexp(r, a.shift);
        } else if (k == edge && before < left) {
            w = we;
        }
        uint64_t incl = w;
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const uint64_t o = __shfl_up(incl, s, 64);
            if (lane >= s) incl += o;
        }
        const uint64_t hit = __ballot(run + incl > target);
        if (hit) {
            if (lane == __ffsll((unsigned long long)hit) - 1) {
                const int64_t n = i + lane;
                winners[b * 4 + 0] = (int32_t)(n / a.HW);
                winners[b * 4 + 1] = tf ? (int32_t)tf[n] : 0;
                winners[b * 4 + 2] = (int32_t)(n % a.HW / a.W);
                winners[b * 4 + 3] = (int32_t)(n % a.HW % a.W);
                n_win[b] = 1;
            }
            return;
        }
        run += __shfl(incl, 63, 64);
        const uint64_t e = __popcll(eqm);
        left -= e < left ? e : left;
    }
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
    a.B = B;
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
    if (dtype == SPK_F32)
        hipLaunchKernelGGL(k_sample_row<float>, dim3((unsigned)B), dim3(THREADS), 0, st,
                           static_cast<const float *>(scores), t_first, u, a, winners, n_winners);
    else
        hipLaunchKernelGGL(k_sample_row<uint16_t>, dim3((unsigned)B), dim3(THREADS), 0, st,
                           static_cast<const uint16_t *>(scores), t_first, u, a, winners, n_winners);
    return spk::check_launch(name);
}
