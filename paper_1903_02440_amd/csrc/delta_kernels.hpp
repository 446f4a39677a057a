// Kernels of the gated delta rule over chunks: the operands of all chunks, and
// the states from chunk to chunk (gfx950).
#pragma once

#include "delta_chunk.hpp"

namespace spk {
namespace delta {

constexpr int LDS_BYTES = 160 * 1024;

// What the operand kernel leaves for the others, per (sequence, key head, chunk)
// and per (sequence, value head, chunk), in bytes:
//   forward   K, K^T, Q        T, coefficients, P
//   backward  K, K^T, Q^T      T, coefficients, T^T, P^T
// The states' kernel reads SCAN_KEY and SCAN_HEAD bytes of each from the start.
template <class E, int DS, bool BWD>
struct Blob : Lay<E, DS> {
    using B = Lay<E, DS>;
    static constexpr int NP = BWD ? 3 : B::NP;
    static constexpr int KEY = BWD ? B::K + 2 * B::KT : 2 * B::K + B::KT;
    static constexpr int T = B::TRI * 3 * FRAG, P = B::TRI * NP * FRAG;
    static constexpr int TTAT = T + B::COEF, PAT = TTAT + (BWD ? T : 0);
    static constexpr int HEAD = PAT + P;
    static constexpr int SCAN_KEY = BWD ? B::K + B::KT : KEY, SCAN_HEAD = BWD ? T + B::COEF : HEAD;
    static constexpr int SCAN = SCAN_KEY + SCAN_HEAD;
};

struct Chunks {
    int NC;               // chunks of the longest sequence
    char *key, *head;     // workspace
};

// What the passes over the chunks keep for the gradients, columns padded to dvp
// (a multiple of 32) and rows to whole chunks and groups of 32 of dk:
//   S, dS  f32 [b * Hv + h][chunk][32 DS][dvp]  state that enters the chunk, gradient of the one that leaves it
//   U, Y   f32 [b * Hv + h][chunk * C][dvp]
struct Kept {
    int dvp;
    float *S, *dS, *U, *Y;
};

// Eight elements of a row of keys or queries, as two runs of four (32 s + 4 g on
// and 16 later), in the row's own type.  Indices past the row are clamped and the
// elements set to 0 by the caller: loads behind a branch would each be waited for.
template <class E>
struct Raw8 {
    E e[8];
};
template <class E, bool WIDE>
__device__ __forceinline__ Raw8<E> load8(const E *p, int s, int g, int dk) {
    Raw8<E> r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int c = 32 * s + 4 * g + 16 * h;
        if constexpr (WIDE) {  // dk a multiple of 4, rows aligned to four elements
            struct alignas(4 * sizeof(E)) Four {
                E e[4];
            };
            const Four w = *reinterpret_cast<const Four *>(p + min(c, dk - 4));
#pragma unroll
            for (int j = 0; j < 4; ++j) r.e[4 * h + j] = w.e[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) r.e[4 * h + j] = p[min(c + j, dk - 1)];
        }
    }
    return r;
}
template <class E>
__device__ __forceinline__ void as_floats(const Raw8<E> &w, int s, int g, int dk, bool row, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = row && 32 * s + slot(g, j) < dk ? to_float(w.e[j]) : 0.0f;
}

constexpr int PREP_THREADS = 256;

// triangular fragment f as (tile of rows, group of summed indices): the lower
// ones of T and P, the upper ones of their transposes
template <int MT, bool UP>
__device__ __forceinline__ void tri_at(int f, int *mt, int *gp) {
    if (MT == 2) {
        *mt = f, *gp = 0;
    } else if (!UP) {
        *mt = f < 2 ? f : 2 + ((f - 2) >> 1), *gp = f < 2 ? 0 : (f - 2) & 1;
    } else {
        *mt = f < 4 ? f >> 1 : f - 2, *gp = f < 4 ? f & 1 : 1;
    }
}

// LDS of the operand kernel: the fragments of K and Q, whose room A and T take
// once the products are made; then the products K K^T and Q K^T.
template <class E, int DS>
struct PrepLds {
    using B = Lay<E, DS>;
    static constexpr int PITCH = B::C + 4;  // floats; 16-byte rows, four banks on from row to row
    static constexpr int SQ = B::C * PITCH * 4;
    static constexpr int R0 = 2 * B::K > 2 * SQ ? 2 * B::K : 2 * SQ;
    static constexpr int BYTES = R0 + 2 * SQ + B::C * 8 + B::C * 4;
};

// Grid (chunk, b * Hk + key head): the fragments of the chunk's keys and
// queries, their products, and for each value head of the key head T, P and the
// coefficients.  T by blocks of 16: the diagonal ones by substitution, a column
// a lane; the rest of block column j by
//     T_ij = -T_ii sum over j <= m < i of A_im T_mj
// on the float matrix cores, a block column a wave.
template <class E, int DS, bool BWD>
__global__ __launch_bounds__(PREP_THREADS) void k_delta_prep(const E *__restrict__ q, const E *__restrict__ k,
                                                             const float *__restrict__ g,
                                                             const float *__restrict__ beta, Args a,
                                                             const int32_t *__restrict__ lengths, int wide, Chunks w) {
    using F = Blob<E, DS, BWD>;
    using S = PrepLds<E, DS>;
    constexpr int C = F::C, MT = F::MT, NT = F::NT, GP = F::GP, PITCH = S::PITCH;
    extern __shared__ char lds[];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, m = lane & 15, gr = lane >> 4;
    const int chunk = blockIdx.x, b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk, rep = a.Hv / a.Hk;
    const int n = (lengths ? max(0, min(a.L, lengths[b])) : a.L) - chunk * C;  // samples from the chunk's first on
    if (n <= 0) return;
    char *fk = lds, *fq = lds + F::K;
    float *A = reinterpret_cast<float *>(lds), *T = A + C * PITCH;
    float *G = reinterpret_cast<float *>(lds + S::R0), *H = G + C * PITCH;
    double *gam = reinterpret_cast<double *>(lds + S::R0 + 2 * S::SQ);
    float *bet = reinterpret_cast<float *>(gam + C);
    char *key = w.key + ((int64_t)blockIdx.y * w.NC + chunk) * F::KEY;

    // K and Q: four units of a thread at a time, so that their loads overlap
    auto units = [&](auto wd) {
        constexpr int NU = 2 * MT * DS * 64 / PREP_THREADS, UB = NU < 4 ? NU : 4;
        for (int u0 = tid; u0 < NU * PREP_THREADS; u0 += UB * PREP_THREADS) {
            Raw8<E> raw[UB];
#pragma unroll
            for (int x = 0; x < UB; ++x) {
                const int f = (u0 + x * PREP_THREADS) >> 6, mt = f / DS % MT, s = f % DS;  // (lane = unit & 63)
                const int i = min(16 * mt + m, n - 1);
                raw[x] = load8<E, decltype(wd)::value>(
                    (f >= MT * DS ? q : k) + (((int64_t)b * a.L + chunk * C + i) * a.Hk + hk) * a.dk, s, gr, a.dk);
            }
#pragma unroll
            for (int x = 0; x < UB; ++x) {
                const int f = (u0 + x * PREP_THREADS) >> 6, mt = f / DS % MT, s = f % DS;
                const bool isq = f >= MT * DS;
                float y[8];
                as_floats(raw[x], s, gr, a.dk, 16 * mt + m < n, y);
                const Terms<NT> t = split<NT>(y);
                const int o = (mt * DS + s) * NT * FRAG;
                put_frag<NT>((isq ? fq : fk) + o, lane, t);
                if (!isq || !BWD) put_frag<NT>(key + (isq ? F::K + F::KT : 0) + o, lane, t);
            }
        }
    };
    if (wide) units(std::true_type{});
    else units(std::false_type{});
    __syncthreads();
    // K^T (and Q^T): row d = 16 t + m, samples slot(gr, j) of group gp
    constexpr int TF = 2 * DS * GP * NT;
    for (int u = tid; u < (BWD ? 2 : 1) * TF * 64; u += PREP_THREADS) {
        const bool isq = u >= TF * 64;
        const int f = (u >> 6) - (isq ? TF : 0), term = f % NT, gp = f / NT % GP, t = f / (NT * GP);
        const char *src = isq ? fq : fk;
        const int d = 16 * t + m, s = d >> 5, r = d & 31, gd = (r & 15) >> 2, jd = (r >> 4) * 4 + (r & 3);
        uint16_t e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = 32 * gp + slot(gr, j);
            e[j] = *reinterpret_cast<const uint16_t *>(src + (((i >> 4) * DS + s) * NT + term) * FRAG +
                                                       (gd * 16 + (i & 15)) * 16 + jd * 2);
        }
        u32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = (uint32_t)e[2 * j] | ((uint32_t)e[2 * j + 1] << 16);
        *reinterpret_cast<u32x4 *>(key + F::K + (isq ? F::KT : 0) + f * FRAG + lane * 16) = o;
    }
    // lower tiles of K K^T (rows 0..MT-1 of the list) and Q K^T (the rest, from the last row on)
    for (int row = wv; row < 2 * MT; row += PREP_THREADS / 64) {
        const bool isq = row >= MT;
        const int mt = isq ? 2 * MT - 1 - row : row;
        const char *fa = isq ? fq : fk;
        for (int nt = 0; nt <= mt; ++nt) {
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < DS; ++s)
                mma<NT, NT>(acc, frag<NT>(fa + (mt * DS + s) * NT * FRAG, lane),
                            frag<NT>(fk + (nt * DS + s) * NT * FRAG, lane));
#pragma unroll
            for (int r = 0; r < 4; ++r) (isq ? H : G)[(16 * mt + 4 * gr + r) * PITCH + 16 * nt + m] = acc[r];
        }
    }
    __syncthreads();  // the fragments' room is free
    for (int hr = 0; hr < rep; ++hr) {
        const int h = hk * rep + hr;
        char *head = w.head + (((int64_t)b * a.Hv + h) * w.NC + chunk) * F::HEAD;
        if (tid < 64) {
            const int64_t at = ((int64_t)b * a.L + chunk * C + tid) * a.Hv + h;
            const bool in = tid < C && tid < n;
            double s = in ? log_decay(g[at]) : 0.0;
#pragma unroll
            for (int o = 1; o < C; o <<= 1) {
                const double p = __shfl_up(s, o, 64);
                if (tid >= o) s += p;
            }
            const double end = __shfl(s, C - 1, 64);
            if (tid < C) {
                const float be = in ? beta[at] : 0.0f;
                gam[tid] = s;
                bet[tid] = be;
                float *co = reinterpret_cast<float *>(head + F::T);
                co[tid] = expf((float)s);
                co[C + tid] = be;
                co[2 * C + tid] = expf((float)(end - s));
                co[3 * C + tid] = a.scale * expf((float)s);
            }
        }
        __syncthreads();
        for (int e = tid; e < C * C; e += PREP_THREADS) {
            const int i = e / C, j = e % C;
            if (j < i) A[i * PITCH + j] = bet[i] * expf((float)(gam[i] - gam[j])) * G[i * PITCH + j];
        }
        for (int u = tid; u < F::TRI * 64; u += PREP_THREADS) {  // P, or P^T
            const int f = u >> 6;
            int mt, gp;
            tri_at<MT, BWD>(f, &mt, &gp);
            const int i = 16 * mt + m;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 32 * gp + slot(gr, j), lo = BWD ? i : c, hi = BWD ? c : i;
                x[j] = lo <= hi ? a.scale * expf((float)(gam[hi] - gam[lo])) * H[hi * PITCH + lo] : 0.0f;
            }
            put_frag<F::NP>(head + F::PAT + f * F::NP * FRAG, lane, split<F::NP>(x));
        }
        __syncthreads();
        if (wv < MT) {  // diagonal block wv, column m (all lane groups alike)
            const float *Ab = A + 16 * wv * PITCH + 16 * wv;
            float x[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float s = i == m ? 1.0f : 0.0f;
#pragma unroll
                for (int j = 0; j < i; ++j) s -= Ab[i * PITCH + j] * x[j];
                x[i] = s;
            }
            if (gr == 0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) T[(16 * wv + i) * PITCH + 16 * wv + m] = x[i];
            }
        }
        __syncthreads();
        if (wv < MT - 1) {  // block column wv
            f32x4 tc[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (i < wv) continue;
                if (i == wv) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) tc[i][r] = T[(16 * i + 4 * gr + r) * PITCH + 16 * i + m];
                    continue;
                }
                f32x4 s = {0.f, 0.f, 0.f, 0.f}, o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < MT; ++c) {
                    if (c < wv || c >= i) continue;
                    const f32x4 al = *reinterpret_cast<const f32x4 *>(A + (16 * i + m) * PITCH + 16 * c + 4 * gr);
#pragma unroll
                    for (int r = 0; r < 4; ++r) s = __builtin_amdgcn_mfma_f32_16x16x4f32(al[r], tc[c][r], s, 0, 0, 0);
                }
                const f32x4 tl = *reinterpret_cast<const f32x4 *>(T + (16 * i + m) * PITCH + 16 * i + 4 * gr);
#pragma unroll
                for (int r = 0; r < 4; ++r) o = __builtin_amdgcn_mfma_f32_16x16x4f32(tl[r], -s[r], o, 0, 0, 0);
                tc[i] = o;
#pragma unroll
                for (int r = 0; r < 4; ++r) T[(16 * i + 4 * gr + r) * PITCH + 16 * wv + m] = o[r];
            }
        }
        __syncthreads();
        for (int u = tid; u < (BWD ? 2 : 1) * F::TRI * 64; u += PREP_THREADS) {  // T (and T^T)
            const bool up = u >= F::TRI * 64;
            const int f = (u >> 6) - (up ? F::TRI : 0);
            int mt, gp;
            if (up) tri_at<MT, true>(f, &mt, &gp);
            else tri_at<MT, false>(f, &mt, &gp);
            const int i = 16 * mt + m;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 32 * gp + slot(gr, j), lo = up ? i : c, hi = up ? c : i;
                x[j] = lo <= hi ? T[hi * PITCH + lo] : 0.0f;
            }
            put_frag<3>(head + (up ? F::TTAT : 0) + f * 3 * FRAG, lane, split<3>(x));
        }
        __syncthreads();
    }
}

// Workgroups go to the eight XCDs in turn; this order puts the value heads of a
// key head, which read the same operands, on one XCD's L2.
__device__ __forceinline__ int head_of(int x, int n) { return n % 8 == 0 ? (x & 7) * (n >> 3) + (x >> 3) : x; }

// Grid (b * Hv + value head, block of columns): a wave carries 16 columns of the
// state through the chunks, in registers: as the right operand of K S and Q S
// (three terms) and as the sums of K^T (last U).  The waves of a workgroup share
// the chunk's operands in LDS and wait for each other only there.  NBUF buffers:
// with two, the next chunk's operands are on their way during this one's products.
// STATES: for the backward pass, the state that enters each chunk and U are
// written instead of out (`kept`).
template <class E, int DS, int NBUF, bool STATES>
__global__ __launch_bounds__(512) void k_delta_scan(const E *__restrict__ v, Args a,
                                                    const int32_t *__restrict__ lengths, int compute, Chunks w,
                                                    const float *state_in, E *__restrict__ out, float *state_out,
                                                    Kept kept) {
    using F = Blob<E, DS, STATES>;
    constexpr int C = F::C, MT = F::MT, NT = F::NT, GP = F::GP, NP = F::NP;
    extern __shared__ char lds[];
    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, gr = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int bh = head_of(blockIdx.x, gridDim.x), b = bh / a.Hv, h = bh % a.Hv, hk = h / (a.Hv / a.Hk);
    const int n = lengths ? max(0, min(a.L, lengths[b])) : a.L, nc = (n + C - 1) / C;
    const int col = ((int)blockIdx.y * compute + wv) * 16 + m;
    const bool mine = wv < compute && col - m < (STATES ? kept.dvp : a.dv), live = mine && col < a.dv;
    const int64_t s0 = (int64_t)bh * a.dk * a.dv + col;
    const char *key = w.key + ((int64_t)b * a.Hk + hk) * w.NC * F::KEY;
    const char *head = w.head + (int64_t)bh * w.NC * F::HEAD;
    f32x4 S[2 * DS];
#pragma unroll
    for (int t = 0; t < 2 * DS; ++t) S[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (state_in) {
        const float *from = state_in + (int64_t)bh * a.dk * a.dv + min(col, a.dv - 1);
#pragma unroll
        for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = from[(int64_t)min(16 * t + 4 * gr + r, a.dk - 1) * a.dv];
#pragma unroll
        for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = live && 16 * t + 4 * gr + r < a.dk ? S[t][r] : 0.0f;
    }
    auto fetch = [&](int c) {
        char *dst = lds + (c % NBUF) * F::SCAN;
        to_lds(dst, key + (int64_t)c * F::KEY, F::SCAN_KEY, wv, waves, lane);
        to_lds(dst + F::SCAN_KEY, head + (int64_t)c * F::HEAD, F::SCAN_HEAD, wv, waves, lane);
    };
    // sample i of the chunk, column col: uniform rows and the lane's offset within four of them
    const int64_t vstep = (int64_t)a.Hv * a.dv;
    const E *vrow = v + ((int64_t)b * a.L * a.Hv + h) * a.dv;
    E *orow = out + ((int64_t)b * a.L * a.Hv + h) * a.dv;
    const uint32_t lin = (uint32_t)((4 * gr * vstep + min(col, a.dv - 1)) * sizeof(E)),
                   lout = (uint32_t)((4 * gr * vstep + col) * sizeof(E));
    E vv[MT][4];
    auto values = [&](int c) {
        const E *p = vrow + (int64_t)c * C * vstep;
        if ((c + 1) * C <= n) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 4; ++r) vv[mt][r] = at(p + (16 * mt + r) * vstep, lin);
        } else {
            // clamped, not skipped: loads behind a branch would each be waited for.  (Rows
            // behind the last sample have beta = 0.)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    vv[mt][r] = p[min(16 * mt + 4 * gr + r, n - 1 - c * C) * vstep + min(col, a.dv - 1)];
        }
    };
    if (nc) {
        values(0);
        fetch(0);
        wait_copies();
    }
    __syncthreads();
    for (int c = 0; c < nc; ++c) {
        float vc[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                vc[mt][r] = to_float(vv[mt][r]);
                if (STATES) vc[mt][r] = live ? vc[mt][r] : 0.0f;  // (the padding is read by others)
            }
        if (c + 1 < nc) {
            values(c + 1);
            if (NBUF == 2) fetch(c + 1);
        }
        f32x4 Y[MT];
        if (mine) {
            const char *K = lds + (c % NBUF) * F::SCAN, *KT = K + F::K, *Q = KT + F::KT, *T = K + F::SCAN_KEY,
                       *P = T + F::PAT;
            const float *co = reinterpret_cast<const float *>(T + F::T);
            if (STATES) {
                float *dst = kept.S + ((int64_t)bh * w.NC + c) * 32 * DS * kept.dvp;
                const uint32_t lo = (uint32_t)(4 * gr * kept.dvp + col) * 4;
#pragma unroll
                for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) at(dst + (16 * t + r) * kept.dvp, lo) = S[t][r];
            }
            f32x4 X[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) X[mt] = Y[mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                const Terms<3> st = split<3>(S[2 * s], S[2 * s + 1]);
                Terms<NP> sp;
#pragma unroll
                for (int i = 0; i < NP; ++i) sp.t[i] = st.t[i];
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mma<NT, 3>(X[mt], frag<NT>(K + (mt * DS + s) * NT * FRAG, lane), st);
                    if (!STATES) mma<NT, NP>(Y[mt], frag<NT>(Q + (mt * DS + s) * NT * FRAG, lane), sp);
                }
            }
            f32x4 U[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const f32x4 ev = *reinterpret_cast<const f32x4 *>(co + 16 * mt + 4 * gr);
                const f32x4 be = *reinterpret_cast<const f32x4 *>(co + C + 16 * mt + 4 * gr);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    X[mt][r] = be[r] * (vc[mt][r] - ev[r] * X[mt][r]);
                }
                U[mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
            }
#pragma unroll
            for (int gp = 0; gp < GP; ++gp) {
                const Terms<3> rt = split<3>(X[2 * gp], X[2 * gp + 1]);
#pragma unroll
                for (int mt = 2 * gp; mt < MT; ++mt) mma<3, 3>(U[mt], frag<3>(T + F::lower(mt, gp) * 3 * FRAG, lane), rt);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                if (!STATES) Y[mt] *= *reinterpret_cast<const f32x4 *>(co + 3 * C + 16 * mt + 4 * gr);
            if (STATES) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) Y[mt] = U[mt];
            }
            const float end = co[C - 1];  // E of the last sample
#pragma unroll
            for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[t][r] *= end;
#pragma unroll
            for (int gp = 0; gp < GP; ++gp) {
                if (!STATES) {
                    const Terms<NP> ut = split<NP>(U[2 * gp], U[2 * gp + 1]);
#pragma unroll
                    for (int mt = 2 * gp; mt < MT; ++mt)
                        mma<NP, NP>(Y[mt], frag<NP>(P + F::lower(mt, gp) * NP * FRAG, lane), ut);
                }
                const f32x4 l0 = *reinterpret_cast<const f32x4 *>(co + 2 * C + 32 * gp + 4 * gr);
                const f32x4 l1 = *reinterpret_cast<const f32x4 *>(co + 2 * C + 32 * gp + 16 + 4 * gr);
                const Terms<3> lt = split<3>(U[2 * gp] * l0, U[2 * gp + 1] * l1);
#pragma unroll
                for (int t = 0; t < 2 * DS; ++t)
                    mma<NT, 3>(S[t], frag<NT>(KT + (t * GP + gp) * NT * FRAG, lane), lt);
            }
        }
        // the next chunk's operands have come; what is stored now has a chunk's time to get out
        if (NBUF == 2) wait_copies();
        __syncthreads();
        if (NBUF == 1 && c + 1 < nc) fetch(c + 1);
        if (STATES && mine) {
            float *dst = kept.U + ((int64_t)bh * w.NC + c) * C * kept.dvp;
            const uint32_t lo = (uint32_t)(4 * gr * kept.dvp + col) * 4;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 4; ++r) at(dst + (16 * mt + r) * kept.dvp, lo) = Y[mt][r];
        }
        if (!STATES && live) {
            E *p = orow + (int64_t)c * C * vstep;
            if ((c + 1) * C <= n) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 4; ++r) at(p + (16 * mt + r) * vstep, lout) = from_float<E>(Y[mt][r]);
            } else {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (c * C + 16 * mt + 4 * gr + r < n) at(p + (16 * mt + r) * vstep, lout) = from_float<E>(Y[mt][r]);
            }
        }
        if (NBUF == 1) {
            wait_copies();
            __syncthreads();
        }
    }
    if (!live || !state_out) return;
#pragma unroll
    for (int t = 0; t < 2 * DS; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = 16 * t + 4 * gr + r;
            if (d < a.dk) state_out[s0 + (int64_t)d * a.dv] = S[t][r];
        }
}

// Waves of a workgroup that carry columns, for `tiles` of 16 columns a head: up
// to eight share the operands, fewer where the workgroups would not fill the CUs.
inline int scan_waves(const Args &a, int tiles) {
    int n = tiles < 8 ? tiles : 8;
    while (n > 1 && (int64_t)a.B * a.Hv * ((tiles + n - 1) / n) < 256) n = (n + 1) / 2;
    return n;
}

inline int groups_of(int dk) {
    const int d = (dk + 31) / 32;
    return d <= 1 ? 1 : d <= 2 ? 2 : d <= 4 ? 4 : 8;
}

#define SPK_DELTA_FORMS(CALL)                     \
    switch (groups_of(a.dk)) {                    \
        case 1: CALL(1);                          \
        case 2: CALL(2);                          \
        case 4: CALL(4);                          \
        default: CALL(8);                         \
    }

// Whether rows of dk elements can be read four at a time.
template <class E>
int wide_rows(int dk, const void *q, const void *k) {
    return dk % 4 == 0 && ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(k)) & (4 * sizeof(E) - 1)) == 0;
}

}  // namespace delta
}  // namespace spk
