// Gradients of the gated delta rule over chunks of samples (gfx950).
//
// With dO the gradient of out and dS that of the state that leaves a chunk, S
// the one that entered it (the other names as in delta_chunk.hpp):
//     dU  = scale P^T dO + last (K dS)       Y = T^T dU
//     dS <- E_C dS + scale Q^T (E dO) - K^T (beta E Y)
// goes from the last chunk to the first, column by column of dv like the
// states.  What is left needs no order, so all chunks do it at once; with
// M = Y U^T (j < i) and N = scale dO U^T (j <= i), both weighed by D:
//     dv    = beta Y
//     dq    = scale E (dO S^T) + N K
//     r     = -E (Y S^T) - M K               the rows of keys, beta apart
//     c     = last (U dS^T) + N^T Q - (beta M)^T K   their columns
//     dk    = beta r + c
//     dbeta_i  = y_i . v_i + k_i . r_i
//     dgamma_i = q_i . dq_i + beta_i k_i . r_i - k_i . c_i, and <dS, S_C> at the end,
// since gamma_i scales q_i and k_i's row by e^gamma_i and k_i's column by its
// inverse; dg is the sum of dgamma from i on.  <dS, S_C> = E_C <dS, S> plus the
// sum of k_j . (last U dS^T)_j.
#include <algorithm>

#include "delta_kernels.hpp"

namespace spk {
namespace delta {

// LDS of the reverse pass: K is needed all through a chunk and has two buffers
// where they fit; Q and the coefficients, T^T and P^T from the middle on.
template <class E, int DS, int KS>
struct RscanLds {
    using F = Blob<E, DS, true>;
    static constexpr int TP = F::HEAD - F::T;  // coefficients, T^T, P^T
    static constexpr int X = KS > 1 ? carriers<DS, KS>() * F::MT * FRAG : 0;
    static constexpr int KB = 3 * F::K + TP + X <= LDS_BYTES ? 2 : 1;
    static constexpr int AT_Q = KB * F::K, AT_TP = AT_Q + F::K, AT_X = AT_TP + TP, BYTES = AT_X + X;
    static_assert(BYTES <= LDS_BYTES, "LDS");
};

// Grid, columns and parts as the states' kernel (delta_kernels.hpp), chunks from
// last to first; the waves of a tile carry 16 columns of dS and add up K dS
// through LDS.  All waves copy here: with some that only copy the others have fewer
// registers, and all gradients of 2 x 1024 samples of 32 memories of 128x128, bfloat16,
// take the same time to 1 us in 265.  Bound as the states' kernel by a chunk's chain,
// 4.7 us for 64 of those samples (2 x 2048: 151 us).
template <class E, int DS, int KS>
__global__ __launch_bounds__(512) void k_delta_rscan(const E *__restrict__ d_out, Args a,
                                                     const int32_t *__restrict__ lengths, int tiles, Chunks w,
                                                     Kept kept, const float *d_last, float *d_first) {
    using F = Blob<E, DS, true>;
    using M = RscanLds<E, DS, KS>;
    constexpr int C = F::C, MT = F::MT, NT = F::NT, GP = F::GP, DW = DS / KS;
    constexpr bool ROOM = DW <= 2;
    constexpr int AHEAD = !ROOM ? 0 : NT == 1 ? 3 : 1, AHEAD3 = ROOM ? 1 : 0;
    extern __shared__ char lds[];
    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, gr = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
    const int tile = wv / KS, part = wv % KS, s0 = part * DW;
    const int bh = head_of(blockIdx.x, gridDim.x), b = bh / a.Hv, h = bh % a.Hv, hk = h / (a.Hv / a.Hk);
    const int n = lengths ? max(0, min(a.L, lengths[b])) : a.L, nc = (n + C - 1) / C;
    const int col = ((int)blockIdx.y * tiles + tile) * 16 + m;
    const bool mine = tile < tiles && col - m < kept.dvp, live = mine && col < a.dv;
    const char *key = w.key + ((int64_t)b * a.Hk + hk) * w.NC * F::KEY;
    const char *head = w.head + (int64_t)bh * w.NC * F::HEAD + F::T;
    f32x4 S[2 * DW];
#pragma unroll
    for (int t = 0; t < 2 * DW; ++t) S[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (d_last) {
        const float *from = d_last + (int64_t)bh * a.dk * a.dv + min(col, a.dv - 1);
#pragma unroll
        for (int t = 0; t < 2 * DW; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = from[(int64_t)min(dk_of(2 * s0 + t, 4 * gr + r), a.dk - 1) * a.dv];
#pragma unroll
        for (int t = 0; t < 2 * DW; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = live && dk_of(2 * s0 + t, 4 * gr + r) < a.dk ? S[t][r] : 0.0f;
    }
    auto fetch_k = [&](int c) { to_lds(lds + (c % M::KB) * F::K, key + (int64_t)c * F::KEY, F::K, wv, waves, lane); };
    auto fetch_rest = [&](int c) {
        to_lds(lds + M::AT_TP, head + (int64_t)c * F::HEAD, M::TP, wv, waves, lane);
        to_lds(lds + M::AT_Q, key + (int64_t)c * F::KEY + F::K, F::K, wv, waves, lane);
    };
    const int64_t vstep = (int64_t)a.Hv * a.dv;
    const E *orow = d_out + ((int64_t)b * a.L * a.Hv + h) * a.dv;
    const uint32_t lin = (uint32_t)((4 * gr * vstep + min(col, a.dv - 1)) * sizeof(E));
    const int ct = (int)blockIdx.y * tiles + tile, vgs = kept.dvp / 32;
    const uint32_t lkept = block_place(ct, lane);
    E on[MT][4];
    auto upstream = [&](int c) {
        const E *p = orow + (int64_t)c * C * vstep;
        if ((c + 1) * C <= n) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 4; ++r) on[mt][r] = at(p + (16 * mt + r) * vstep, lin);
        } else {  // (clamped, not skipped: loads behind a branch would each be waited for)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    on[mt][r] = p[min(16 * mt + 4 * gr + r, n - 1 - c * C) * vstep + min(col, a.dv - 1)];
        }
    };
    if (nc) {
        upstream(nc - 1);
        fetch_k(nc - 1);
        wait_copies();
        fetch_rest(nc - 1);
    }
    __syncthreads();
    for (int c = nc - 1; c >= 0; --c) {
        const char *K = lds + (c % M::KB) * F::K, *Q = lds + M::AT_Q, *H = lds + M::AT_TP;
        const char *TT = H + (F::TTAT - F::T), *PT = H + (F::PAT - F::T);
        const float *co = reinterpret_cast<const float *>(H);
        f32x4 X[MT], Y[MT];
        if (mine) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) X[mt] = Y[mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
            Terms<3> st;
            stream<DW * MT, AHEAD>([&](int i) { return frag<NT>(K + (i % MT * DS + s0 + i / MT) * NT * FRAG, lane); },
                                   [&](int i, const Terms<NT> &f) {
                                       const int s = i / MT;
                                       if (i % MT == 0) st = split<3>(S[2 * s], S[2 * s + 1]);
                                       mma<NT, 3>(X[i % MT], f, st);
                                   });
            if (KS > 1) {
                char *xb = lds + M::AT_X + tile * KS * MT * FRAG;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    *reinterpret_cast<f32x4 *>(xb + (part * MT + mt) * FRAG + lane * 16) = X[mt];
            }
        }
        wait_copies();  // what the second half needs of this chunk
        lds_barrier();
        float o[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                o[mt][r] = live && c * C + 16 * mt + 4 * gr + r < n ? to_float(on[mt][r]) : 0.0f;
                made(o[mt][r]);
            }
        if (c > 0) {
            upstream(c - 1);
            if (M::KB == 2) fetch_k(c - 1);
        }
        if (mine) {
            if (KS > 1) {
                const char *xb = lds + M::AT_X + tile * KS * MT * FRAG;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    f32x4 x[KS];
#pragma unroll
                    for (int p = 0; p < KS; ++p) x[p] = *reinterpret_cast<const f32x4 *>(xb + (p * MT + mt) * FRAG + lane * 16);
#pragma unroll
                    for (int p = 1; p < KS; ++p) x[0] += x[p];
                    X[mt] = x[0];
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)  // dU: last (K dS), and P^T dO on top
                X[mt] *= *reinterpret_cast<const f32x4 *>(co + 2 * C + 16 * mt + 4 * gr);
            // fragments of P^T, then of T^T: columns of 32 samples, above the diagonal
            Terms<NT> ot;
            Terms<3> ut;
            stream<2 * F::TRI, AHEAD3>(
                [&](int i) {
                    const int f = i % F::TRI, gp = f < 2 ? 0 : 1, mt = f < 2 ? f : f - 2;
                    return frag<3>((i < F::TRI ? PT : TT) + F::upper(mt, gp) * 3 * FRAG, lane);
                },
                [&](int i, const Terms<3> &fr) {
                    const int f = i % F::TRI, gp = f < 2 ? 0 : 1, mt = f < 2 ? f : f - 2;
                    if (i < F::TRI) {
                        if (mt == 0) {
                            float x[8];
#pragma unroll
                            for (int j = 0; j < 8; ++j) x[j] = o[2 * gp + (j >> 2)][j & 3];
                            ot = split<NT>(x);
                        }
                        mma<3, NT>(X[mt], fr, ot);
                    } else {
                        if (mt == 0) ut = split<3>(X[2 * gp], X[2 * gp + 1]);
                        mma<3, 3>(Y[mt], fr, ut);
                    }
                });
            // (here, so that they have the rest of the chunk to get out before a wait)
            f32x4 *dst = kept.dS + ((((int64_t)bh * w.NC + c) * 2 * DS + 2 * s0) * vgs + (ct >> 1)) * KEPT_BLOCK;
#pragma unroll
            for (int t = 0; t < 2 * DW; ++t) at(dst + t * vgs * KEPT_BLOCK, lkept) = quad_transpose(S[t], lane);
            const float end = co[C - 1];
#pragma unroll
            for (int t = 0; t < 2 * DW; ++t) S[t] *= end;
#pragma unroll
            for (int gp = 0; gp < GP; ++gp) {
                float x[8], y[8];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const f32x4 ev = *reinterpret_cast<const f32x4 *>(co + 32 * gp + 16 * hf + 4 * gr);
                    const f32x4 be = *reinterpret_cast<const f32x4 *>(co + C + 32 * gp + 16 * hf + 4 * gr);
                    const f32x4 es = *reinterpret_cast<const f32x4 *>(co + 3 * C + 32 * gp + 16 * hf + 4 * gr);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        x[4 * hf + r] = es[r] * o[2 * gp + hf][r];
                        y[4 * hf + r] = -be[r] * ev[r] * Y[2 * gp + hf][r];
                    }
                }
                const Terms<3> xt = split<3>(x), yt = split<3>(y);
                stream<4 * DW, AHEAD>([&](int i) { return tfrag<NT, DS>(i & 1 ? K : Q, 2 * s0 + i / 2, gp, lane); },
                                      [&](int i, const Terms<NT> &f) { mma<NT, 3>(S[i / 2], f, i & 1 ? yt : xt); });
            }
        }
        wait_copies();
        lds_barrier();
        if (c > 0 && M::KB == 1) fetch_k(c - 1);
        if (M::KB == 1) {
            wait_copies();
            lds_barrier();
        }
        if (c > 0) fetch_rest(c - 1);
        if (mine) {
            f32x4 *yd = kept.Y + (((int64_t)bh * w.NC + c) * MT * vgs + (ct >> 1)) * KEPT_BLOCK;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                if (part == mt * KS / MT) at(yd + mt * vgs * KEPT_BLOCK, lkept) = quad_transpose(Y[mt], lane);
        }
    }
    if (!live || !d_first) return;
#pragma unroll
    for (int t = 0; t < 2 * DW; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = dk_of(2 * s0 + t, 4 * gr + r);
            if (d < a.dk) d_first[(int64_t)bh * a.dk * a.dv + (int64_t)d * a.dv + col] = S[t][r];
        }
}

// Eight neighbouring elements of a row as they were loaded: taken apart only where
// they are used, since taking them apart waits for them.  WIDE: rows of dv elements
// go four at a time.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <class E, bool WIDE>
struct Eight {
    E e[8];
    __device__ __forceinline__ void load(const E *row, int c, int dv) {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = row[min(c + j, dv - 1)];
    }
    __device__ __forceinline__ float get(int j) const { return to_float(e[j]); }
    static __device__ __forceinline__ void store(E *row, int c, int dv, const float (&x)[8]) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < dv) row[c + j] = from_float<E>(x[j]);
    }
};
template <>
struct Eight<float, true> {
    f32x4 e[2];
    __device__ __forceinline__ void load(const float *row, int c, int dv) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) e[hf] = *reinterpret_cast<const f32x4 *>(row + min(c + 4 * hf, dv - 4));
    }
    __device__ __forceinline__ float get(int j) const { return e[j >> 2][j & 3]; }
    static __device__ __forceinline__ void store(float *row, int c, int dv, const float (&x)[8]) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
            if (c + 4 * hf < dv)
                *reinterpret_cast<f32x4 *>(row + c + 4 * hf) = (f32x4){x[4 * hf], x[4 * hf + 1], x[4 * hf + 2], x[4 * hf + 3]};
    }
};
template <>
struct Eight<uint16_t, true> {
    u32x2 e[2];
    __device__ __forceinline__ void load(const uint16_t *row, int c, int dv) {
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) e[hf] = *reinterpret_cast<const u32x2 *>(row + min(c + 4 * hf, dv - 4));
    }
    __device__ __forceinline__ float get(int j) const {
        const uint32_t w = e[j >> 2][(j >> 1) & 1];
        return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
    }
    static __device__ __forceinline__ void store(uint16_t *row, int c, int dv, const float (&x)[8]) {
        auto two = [](float lo, float hi) {
            return (uint32_t)from_float<uint16_t>(lo) | ((uint32_t)from_float<uint16_t>(hi) << 16);
        };
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
            if (c + 4 * hf < dv)
                *reinterpret_cast<u32x2 *>(row + c + 4 * hf) =
                    (u32x2){two(x[4 * hf], x[4 * hf + 1]), two(x[4 * hf + 2], x[4 * hf + 3])};
    }
};

constexpr int GRAD_WAVES = 8, GRAD_THREADS = GRAD_WAVES * 64;

template <class E, int DS>
struct GradLds {
    using B = Lay<E, DS>;
    static constexpr int PITCH = B::C + 4, SQ = B::C * PITCH * 4;
    static constexpr int ONE = B::MT * (B::NT + 6) * FRAG;  // dO, Y, U of 32 columns
    static constexpr int TRI = B::TRI * 3 * FRAG;           // N, M, N^T, (beta M)^T: four of these
    static constexpr int SUMS = (2 * GRAD_WAVES + 1) * B::C * 4 + GRAD_WAVES * 4;
    // M and N as floats take the room of the staged columns
    static constexpr int TEMP = ONE > 2 * SQ ? ONE : 2 * SQ;
    // K and Q, all of their groups of 32 of dk where they fit, else those of one pass of the waves
    static constexpr bool WHOLE = TEMP + 2 * B::K + 4 * TRI + SUMS + 8192 <= LDS_BYTES;
    static constexpr int GROUPS = WHOLE ? DS : GRAD_WAVES / 2, K = B::MT * GROUPS * B::NT * FRAG, KQ = 2 * K;
    static constexpr int AT_KQ = TEMP, AT_TRI = AT_KQ + KQ, AT_SUMS = AT_TRI + 4 * TRI;
    static constexpr int AT_GAM = AT_SUMS + (SUMS + 15) / 16 * 16, BYTES = AT_GAM + B::C * 8 + 3 * B::C * 4;
};

// Grid (chunk, b * Hk + key head): everything of the list above that has no
// order.  A wave owns 16 of the dk columns of dq, r and c (every eighth tile);
// the sums over dv go by groups of 32 columns whose fragments all waves share,
// and the tiles of M and N are dealt out among the waves.  The value heads of a
// key head follow each other, so that their dq and dk add up in registers.  The LDS
// (144 KB at 128 rows, bfloat16) leaves one workgroup a CU, whose eight waves wait for
// each other between short steps: the matrix cores are busy 18 % of the time.
// 2 x 2048 samples of 16 keys for 32 heads of 128x128: 225 us, 2.6 TB/s.
template <class E, int DS, bool WIDE>
__global__ __launch_bounds__(GRAD_THREADS) void k_delta_grads(
    const E *__restrict__ v, const float *__restrict__ g, const E *__restrict__ d_out, Args a,
    const int32_t *__restrict__ lengths, Chunks w, Kept kept, E *__restrict__ d_q,
    E *__restrict__ d_k, E *__restrict__ d_v, float *__restrict__ d_g, float *__restrict__ d_beta) {
    using F = Blob<E, DS, true>;
    using G = GradLds<E, DS>;
    constexpr int C = F::C, MT = F::MT, NT = F::NT, GP = F::GP, PITCH = G::PITCH;
    constexpr int TW = (2 * DS + GRAD_WAVES - 1) / GRAD_WAVES;  // dk tiles of a wave
    constexpr int LT = MT * (MT + 1) / 2, LW = (2 * LT + GRAD_WAVES - 1) / GRAD_WAVES;  // tiles of M and N
    static_assert(2 * MT <= GRAD_WAVES, "a wave a tile of Y and of U");
    extern __shared__ char lds[];
    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, gr = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int chunk = blockIdx.x, b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk, rep = a.Hv / a.Hk;
    const int n = (lengths ? max(0, min(a.L, lengths[b])) : a.L) - chunk * C;
    if (n <= 0) return;
    char *fo = lds, *fy = fo + MT * NT * FRAG, *fu = fy + MT * 3 * FRAG;
    float *sqM = reinterpret_cast<float *>(lds), *sqN = sqM + C * PITCH;
    char *tri = lds + G::AT_TRI;  // N, M, N^T, (beta M)^T
    float *sums = reinterpret_cast<float *>(lds + G::AT_SUMS);  // [waves][2][C], then y.v; then the ends
    float *yv = sums + 2 * GRAD_WAVES * C, *ends = yv + C;
    double *gam = reinterpret_cast<double *>(lds + G::AT_GAM);
    float *co = reinterpret_cast<float *>(gam + C);  // E, beta, last
    const char *key = w.key + ((int64_t)blockIdx.y * w.NC + chunk) * F::KEY;
    const int64_t row0 = (int64_t)b * a.L + chunk * C;

    const char *fk = lds + G::AT_KQ, *fq = fk + G::K;
    // groups of dk from s0 on of K and Q
    auto fetch = [&](int s0) {
        if (G::WHOLE) {
            to_lds(lds + G::AT_KQ, key, G::KQ, wv, GRAD_WAVES, lane);
        } else {
#pragma unroll
            for (int x = 0; x < 2 * MT; ++x)  // K's tiles of samples, then Q's
                to_lds(lds + G::AT_KQ + x * G::GROUPS * NT * FRAG, key + (x * DS + s0) * NT * FRAG, G::GROUPS * NT * FRAG, wv,
                       GRAD_WAVES, lane);
        }
    };
    if (G::WHOLE) fetch(0);

    f32x4 dqs[TW][MT], dks[TW][MT];
#pragma unroll
    for (int p = 0; p < TW; ++p)
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) dqs[p][mt] = dks[p][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};

    for (int hr = 0; hr < rep; ++hr) {
        const int h = hk * rep + hr;
        const int64_t bh = (int64_t)b * a.Hv + h, ch = bh * w.NC + chunk;
        const float *cog = reinterpret_cast<const float *>(w.head + ch * F::HEAD + F::T);
        const int vgs = kept.dvp / 32;
        const f32x4 *S = kept.S + ch * 2 * DS * vgs * KEPT_BLOCK, *dS = kept.dS + ch * 2 * DS * vgs * KEPT_BLOCK;
        const f32x4 *U = kept.U + ch * MT * vgs * KEPT_BLOCK, *Y = kept.Y + ch * MT * vgs * KEPT_BLOCK;
        f32x4 dq[TW][MT], rr[TW][MT], cc[TW][MT], mn[LW];
#pragma unroll
        for (int p = 0; p < TW; ++p)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) dq[p][mt] = rr[p][mt] = cc[p][mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int l = 0; l < LW; ++l) mn[l] = (f32x4){0.f, 0.f, 0.f, 0.f};
        float dot = 0.0f;   // <dS, S>, the lane's part
        float yvp = 0.0f;   // y.v of row 16 wv + m, the lane's part (waves below MT)
        // The wave's share of the next 32 columns is on its way while these are used:
        // a tile of samples of Y (wave mt) or U (wave MT + mt), with v beside Y and dO
        // beside U, and the rows of S and dS that are its right operands.  No load
        // depends on a branch: it would be waited for where the branches meet.
        const bool of_u = wv >= MT, stages = wv < 2 * MT;
        const int mt0 = wv % MT, i0 = 16 * mt0 + m;
        const f32x4 *yu_from = (of_u ? U : Y) + mt0 * vgs * KEPT_BLOCK + lane;
        const E *vo_from = (of_u ? d_out : v) + ((row0 + min(i0, n - 1)) * a.Hv + h) * a.dv;
        f32x4 sn[TW][2], en[TW][2], yu[2];
        Eight<E, WIDE> vo;
        auto load_states = [&](int vg) {
#pragma unroll
            for (int p = 0; p < TW; ++p) {
                const int t = min(p * GRAD_WAVES + wv, 2 * DS - 1);
                const int at = (t * vgs + vg) * KEPT_BLOCK + lane;
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    sn[p][hf] = S[at + 64 * hf];
                    en[p][hf] = dS[at + 64 * hf];
                }
            }
        };
        auto load = [&](int vg) {
            if (TW == 1) load_states(vg);  // (two tiles a wave have no registers to spare for it)
            yu[0] = yu_from[vg * KEPT_BLOCK];
            yu[1] = yu_from[vg * KEPT_BLOCK + 64];
            vo.load(vo_from, 32 * vg + 8 * gr, a.dv);
        };
        load(0);
        if (tid < 64) {
            double s = tid < C && tid < n ? log_decay(g[(row0 + tid) * a.Hv + h]) : 0.0;
#pragma unroll
            for (int o = 1; o < C; o <<= 1) {
                const double p = __shfl_up(s, o, 64);
                if (tid >= o) s += p;
            }
            if (tid < C) gam[tid] = s;
        }
        for (int i = tid; i < 3 * C; i += GRAD_THREADS) co[i] = cog[i];
        for (int vg = 0; vg < kept.dvp / 32; ++vg) {
            __syncthreads();  // the staged columns (and, at first, the coefficients) may be written
            if (stages) {
                const int cv = 32 * vg + 8 * gr;
                const float y[8] = {yu[0][0], yu[0][1], yu[0][2], yu[0][3], yu[1][0], yu[1][1], yu[1][2], yu[1][3]};
                float x[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = i0 < n && cv + j < a.dv ? vo.get(j) : 0.0f;
                put_frag<3>((of_u ? fu : fy) + mt0 * 3 * FRAG, lane, split<3, true>(y));
                if (of_u) {
                    put_frag<NT>(fo + mt0 * NT * FRAG, lane, split<NT, true>(x));
                } else {
                    const float be = co[C + i0];
                    float d[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        yvp += cv + j < a.dv && i0 < n ? y[j] * x[j] : 0.0f;
                        d[j] = be * y[j];
                    }
                    if (i0 < n) Eight<E, WIDE>::store(d_v + ((row0 + i0) * a.Hv + h) * a.dv, cv, a.dv, d);
                }
            }
            if (TW > 1) load_states(vg);
            f32x4 sc[TW][2], ec[TW][2];
#pragma unroll
            for (int p = 0; p < TW; ++p)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) sc[p][hf] = sn[p][hf], ec[p][hf] = en[p][hf];
            __syncthreads();
            if (vg + 1 < kept.dvp / 32) load(vg + 1);
#pragma unroll
            for (int p = 0; p < TW; ++p) {
                const int t = p * GRAD_WAVES + wv;
                if (t >= 2 * DS) continue;
#pragma unroll
                for (int r = 0; r < 4; ++r) dot += sc[p][0][r] * ec[p][0][r] + sc[p][1][r] * ec[p][1][r];
                const Terms<3> st = split<3>(sc[p][0], sc[p][1]), et = split<3>(ec[p][0], ec[p][1]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    mma<NT, 3>(dq[p][mt], frag<NT>(fo + mt * NT * FRAG, lane), st);
                    mma<3, 3>(rr[p][mt], frag<3>(fy + mt * 3 * FRAG, lane), st);
                    mma<3, 3>(cc[p][mt], frag<3>(fu + mt * 3 * FRAG, lane), et);
                }
            }
#pragma unroll
            for (int l = 0; l < LW; ++l) {
                const int idx = l * GRAD_WAVES + wv;
                if (idx >= 2 * LT) continue;
                int mt = 0, nt = idx % LT;
                while (nt > mt) nt -= ++mt;
                if (idx < LT) mma<3, 3>(mn[l], frag<3>(fy + mt * 3 * FRAG, lane), frag<3>(fu + nt * 3 * FRAG, lane));
                else mma<NT, 3>(mn[l], frag<NT>(fo + mt * NT * FRAG, lane), frag<3>(fu + nt * 3 * FRAG, lane));
            }
        }
        __syncthreads();  // the staged columns are done with
#pragma unroll
        for (int l = 0; l < LW; ++l) {
            const int idx = l * GRAD_WAVES + wv;
            if (idx >= 2 * LT) continue;
            int mt = 0, nt = idx % LT;
            while (nt > mt) nt -= ++mt;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * mt + 4 * gr + r, j = 16 * nt + m;
                const float d = j <= i ? expf((float)(gam[i] - gam[j])) : 0.0f;
                if (idx < LT) sqM[i * PITCH + j] = j < i ? d * mn[l][r] : 0.0f;
                else sqN[i * PITCH + j] = a.scale * d * mn[l][r];
            }
        }
        if (wv < MT) {
            yvp += __shfl_xor(yvp, 16, 64);
            yvp += __shfl_xor(yvp, 32, 64);
            if (gr == 0) yv[16 * wv + m] = yvp;
        }
#pragma unroll
        for (int s = 32; s >= 1; s >>= 1) dot += __shfl_xor(dot, s, 64);
        if (lane == 0) ends[wv] = co[C - 1] * dot;
        __syncthreads();
        for (int u = tid; u < 4 * F::TRI * 64; u += GRAD_THREADS) {
            const int f4 = u >> 6, which = f4 / F::TRI, f = f4 % F::TRI;  // N, M, N^T, (beta M)^T
            int mt, gp;
            if (which < 2) tri_at<MT, false>(f, &mt, &gp);
            else tri_at<MT, true>(f, &mt, &gp);
            const int i = 16 * mt + m;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 32 * gp + slot(gr, j), lo = which < 2 ? c : i, hi = which < 2 ? i : c;
                x[j] = lo <= hi ? (which & 1 ? sqM : sqN)[hi * PITCH + lo] : 0.0f;
                if (which == 3) x[j] *= co[C + hi];
            }
            put_frag<3>(tri + which * G::TRI + f * 3 * FRAG, lane, split<3>(x));
        }
        __syncthreads();
        if (G::WHOLE && hr == 0) {  // K and Q have come
            wait_copies();
            lds_barrier();
        }
        float pg[MT][4], pb[MT][4], pe = 0.0f;  // row sums: dgamma, k.r; k.(last U dS^T) of all rows
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r) pg[mt][r] = pb[mt][r] = 0.0f;
#pragma unroll
        for (int p = 0; p < TW; ++p) {
            const int t = p * GRAD_WAVES + wv, tl = G::WHOLE ? t : wv;  // (tl: in what LDS has of K and Q)
            if (!G::WHOLE) {
                lds_barrier();
                fetch(p * G::GROUPS);
                wait_copies();
                lds_barrier();
            }
            if (t >= 2 * DS) continue;
            Terms<NT> kt[GP], qt[GP];
#pragma unroll
            for (int gp = 0; gp < GP; ++gp) {
                kt[gp] = tfrag<NT, G::GROUPS>(fk, tl, gp, lane);
                qt[gp] = tfrag<NT, G::GROUPS>(fq, tl, gp, lane);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const f32x4 ev = *reinterpret_cast<const f32x4 *>(co + 16 * mt + 4 * gr);
                const f32x4 be = *reinterpret_cast<const f32x4 *>(co + C + 16 * mt + 4 * gr);
                const f32x4 la = *reinterpret_cast<const f32x4 *>(co + 2 * C + 16 * mt + 4 * gr);
                f32x4 x = a.scale * ev * dq[p][mt], y = (f32x4){0.f, 0.f, 0.f, 0.f} - ev * rr[p][mt], z = la * cc[p][mt];
                float kk[4], qq[4];  // k and q at the tile's places
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    kk[r] = qq[r] = 0.0f;
#pragma unroll
                    for (int x = 0; x < NT; ++x) {
                        const int o = ((mt * G::GROUPS + (tl >> 1)) * NT + x) * FRAG +
                                      ((m >> 2) * 16 + 4 * gr + r) * 16 + (4 * (tl & 1) + (m & 3)) * 2;
                        kk[r] += to_float(*reinterpret_cast<const uint16_t *>(fk + o));
                        qq[r] += to_float(*reinterpret_cast<const uint16_t *>(fq + o));
                    }
                    pe += kk[r] * z[r];
                }
                f32x4 mk = {0.f, 0.f, 0.f, 0.f}, mc = mk;
#pragma unroll
                for (int gp = 0; gp < GP; ++gp) {
                    if (gp <= mt / 2) {
                        mma<3, NT>(x, frag<3>(tri + F::lower(mt, gp) * 3 * FRAG, lane), kt[gp]);
                        mma<3, NT>(mk, frag<3>(tri + G::TRI + F::lower(mt, gp) * 3 * FRAG, lane), kt[gp]);
                    }
                    if (gp >= mt / 2) {
                        mma<3, NT>(z, frag<3>(tri + 2 * G::TRI + F::upper(mt, gp) * 3 * FRAG, lane), qt[gp]);
                        mma<3, NT>(mc, frag<3>(tri + 3 * G::TRI + F::upper(mt, gp) * 3 * FRAG, lane), kt[gp]);
                    }
                }
                y -= mk;
                z -= mc;
                dqs[p][mt] += x;
                dks[p][mt] += be * y + z;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    pb[mt][r] += kk[r] * y[r];
                    pg[mt][r] += qq[r] * x[r] + be[r] * (kk[r] * y[r]) - kk[r] * z[r];
                }
            }
        }
        // Sums over the 16 lanes of a row group: at each step a lane keeps one half of its
        // values and gives the other away.
        constexpr int NV = 8 * MT;
        float x[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = i & 1 ? pb[i >> 3][(i >> 1) & 3] : pg[i >> 3][(i >> 1) & 3];
#pragma unroll
        for (int s = 8, half = NV / 2; s >= 1; s >>= 1, half >>= 1)
#pragma unroll
            for (int i = 0; i < half; ++i) {
                const bool up = m & s;
                const float give = up ? x[i] : x[i + half];
                x[i] = (up ? x[i + half] : x[i]) + __shfl_xor(give, s, 64);
            }
#pragma unroll
        for (int j = 0; j < NV / 16; ++j) {
            const int i = m * (NV / 16) + j;
            sums[(2 * wv + (i & 1)) * C + 16 * (i >> 3) + 4 * gr + ((i >> 1) & 3)] = x[j];
        }
#pragma unroll
        for (int s = 32; s >= 1; s >>= 1) pe += __shfl_xor(pe, s, 64);
        if (lane == 0) ends[wv] += pe;
        __syncthreads();
        if (tid < 64) {
            double x = 0.0;
            float y = tid < C ? yv[tid] : 0.0f;
            for (int q8 = 0; q8 < GRAD_WAVES; ++q8) {
                if (tid < C) {
                    x += sums[2 * q8 * C + tid];
                    y += sums[(2 * q8 + 1) * C + tid];
                }
                if (tid == C - 1) x += ends[q8];
            }
#pragma unroll
            for (int o = 1; o < C; o <<= 1) {  // the sum from tid on
                const double p = __shfl_down(x, o, 64);
                if (tid + o < C) x += p;
            }
            if (tid < C && tid < n) {
                d_g[(row0 + tid) * a.Hv + h] = (float)x;
                d_beta[(row0 + tid) * a.Hv + h] = y;
            }
        }
        __syncthreads();  // gam, co and the sums are written again
    }
#pragma unroll
    for (int p = 0; p < TW; ++p) {
        const int t = p * GRAD_WAVES + wv, d = dk_of(t, m);
        if (t >= 2 * DS || d >= a.dk) continue;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * mt + 4 * gr + r;
                if (i >= n) continue;
                const int64_t at = ((row0 + i) * a.Hk + hk) * a.dk + d;
                d_q[at] = from_float<E>(dqs[p][mt][r]);
                d_k[at] = from_float<E>(dks[p][mt][r]);
            }
    }
}

namespace {

template <class E, int DS>
size_t carve(void *ws, const Args &a, Chunks *w, Kept *kept) {
    using F = Blob<E, DS, true>;
    spk::Carver c(ws);
    const size_t bh = (size_t)a.B * a.Hv;
    w->NC = (a.L + F::C - 1) / F::C;
    kept->dvp = (a.dv + 31) / 32 * 32;
    w->key = c.take<char>((size_t)a.B * a.Hk * w->NC * F::KEY);
    w->head = c.take<char>(bh * w->NC * F::HEAD);
    kept->S = c.take<f32x4>(bh * w->NC * 8 * DS * kept->dvp);
    kept->dS = c.take<f32x4>(bh * w->NC * 8 * DS * kept->dvp);
    kept->U = c.take<f32x4>(bh * w->NC * F::C / 4 * kept->dvp);
    kept->Y = c.take<f32x4>(bh * w->NC * F::C / 4 * kept->dvp);
    return spk::align_up(c.off, 256);
}

template <class E, int DS, int KS>
void launch_rscan(const Cols &cols, const E *d_out, const Args &a, const int32_t *lengths, const Chunks &w,
                  const Kept &kept, const float *d_last, float *d_first, hipStream_t st) {
    constexpr int LDS = RscanLds<E, DS, KS>::BYTES;
    hipLaunchKernelGGL((k_delta_rscan<E, DS, KS>), dim3((unsigned)(a.B * a.Hv), (unsigned)cols.blocks),
                       dim3(64 * std::max(4, cols.tiles * KS)), LDS, st, d_out, a, lengths, cols.tiles, w, kept, d_last, d_first);
}

struct Call {
    const void *q, *k, *v;
    const float *g, *beta;
    const int32_t *lengths;
    const float *state_in;
    const void *d_out;
    const float *d_last;
    void *d_q, *d_k, *d_v;
    float *d_g, *d_beta, *d_first;
};

template <class E, int DS>
int backward(const Call &c, const Args &a, void *ws, hipStream_t st, const char *name) {
    constexpr int LP = PrepLds<E, DS>::BYTES, LG = GradLds<E, DS>::BYTES;
    Chunks w;
    Kept kept;
    carve<E, DS>(ws, a, &w, &kept);
    const E *q = static_cast<const E *>(c.q), *k = static_cast<const E *>(c.k), *v = static_cast<const E *>(c.v);
    const E *d_out = static_cast<const E *>(c.d_out);
    const dim3 per_key((unsigned)w.NC, (unsigned)(a.B * a.Hk));
    hipLaunchKernelGGL((k_delta_prep<E, DS, true>), per_key, dim3(PREP_THREADS), LP, st, q, k, c.g, c.beta, a,
                       c.lengths, wide_rows<E>(a.dk, q, k), w);
    static_assert(LP <= LDS_BYTES && LG <= LDS_BYTES, "LDS");
    const Cols cols = columns(a, kept.dvp / 16, DS);
#define SPK_SCAN(KS)                                                                                                \
    launch_scan<E, DS, KS, true>(cols, v, a, c.lengths, w, c.state_in, nullptr, nullptr, kept, st);                 \
    launch_rscan<E, DS, KS>(cols, d_out, a, c.lengths, w, kept, c.d_last, c.d_first, st)
    SPK_DELTA_PARTS(DS, cols, SPK_SCAN)
#undef SPK_SCAN
    const bool fours = ((reinterpret_cast<uintptr_t>(c.v) | reinterpret_cast<uintptr_t>(c.d_out) |
                         reinterpret_cast<uintptr_t>(c.d_v)) & (4 * sizeof(E) - 1)) == 0;
#define SPK_GRADS(WIDE)                                                                                             \
    hipLaunchKernelGGL((k_delta_grads<E, DS, WIDE>), per_key, dim3(GRAD_THREADS), LG, st, v, c.g, d_out, a, c.lengths, w, \
                       kept, static_cast<E *>(c.d_q), static_cast<E *>(c.d_k), static_cast<E *>(c.d_v), c.d_g, c.d_beta)
    if (a.dv % 4 == 0 && fours) SPK_GRADS(true);
    else SPK_GRADS(false);
#undef SPK_GRADS
    return spk::check_launch(name);
}

size_t workspace_bytes(const Args &a) {
    Chunks w;
    Kept kept;
#define SPK_WS(DS) \
    return a.dtype == SPK_F32 ? carve<float, DS>(nullptr, a, &w, &kept) : carve<uint16_t, DS>(nullptr, a, &w, &kept)
    SPK_DELTA_FORMS(SPK_WS)
#undef SPK_WS
}

int run(const Call &c, const Args &a, void *ws, hipStream_t st, const char *name) {
#define SPK_BW(DS) \
    return a.dtype == SPK_F32 ? backward<float, DS>(c, a, ws, st, name) : backward<uint16_t, DS>(c, a, ws, st, name)
    SPK_DELTA_FORMS(SPK_BW)
#undef SPK_BW
}

// No samples: the gradient passes through.
__global__ __launch_bounds__(256) void k_pass(const float *src, float *dst, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256)
        dst[i] = src ? src[i] : 0.0f;
}

}  // namespace
}  // namespace delta
}  // namespace spk

using namespace spk::delta;

extern "C" size_t spk_delta_rule_backward_workspace_size(int dtype, int B, int L, int Hk, int Hv, int dk, int dv) {
    const Args a{dtype, B, L, Hk, Hv, dk, dv, 1.0f};
    return check(a, "") == SPK_OK && B > 0 && L > 0 ? workspace_bytes(a) : 0;
}

extern "C" int spk_delta_rule_backward(const void *q, const void *k, const void *v, const float *g, const float *beta,
                                       int dtype, int B, int L, int Hk, int Hv, int dk, int dv, float scale,
                                       const int32_t *lengths, const float *initial_state, const void *d_out,
                                       const float *d_final_state, void *d_q, void *d_k, void *d_v, float *d_g,
                                       float *d_beta, float *d_initial_state, void *workspace, size_t ws_bytes,
                                       void *stream) {
    const char *name = "spk_delta_rule_backward";
    const Args a{dtype, B, L, Hk, Hv, dk, dv, scale};
    if (int rc = check(a, name)) return rc;
    if (B == 0) return spk::ok();
    hipStream_t st = spk::as_stream(stream);
    if (L == 0) {
        if (!d_initial_state) return spk::ok();
        const int64_t n = (int64_t)B * Hv * dk * dv;
        hipLaunchKernelGGL(k_pass, dim3((unsigned)std::min<int64_t>(4096, spk::ceil_div(n, 256))), dim3(256), 0, st,
                           d_final_state, d_initial_state, n);
        return spk::check_launch(name);
    }
    SPK_REQUIRE(q && k && v && g && beta && d_out && d_q && d_k && d_v && d_g && d_beta, SPK_E_ARG,
                "%s: all inputs, d_out and the gradients d_q, d_k, d_v, d_g and d_beta are required", name);
    const size_t need = workspace_bytes(a);
    SPK_REQUIRE(workspace && ws_bytes >= need, SPK_E_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", name,
                workspace ? ws_bytes : (size_t)0, need);
    SPK_REQUIRE(aligned16(workspace), SPK_E_ARG, "%s: the workspace must be 16-byte aligned", name);
    const Call c{q, k, v, g, beta, lengths, initial_state, d_out, d_final_state, d_q, d_k, d_v, d_g, d_beta,
                 d_initial_state};
    return run(c, a, workspace, st, name);
}
