// Kernels of the gated delta rule over chunks: the operands of all chunks, and
// the states from chunk to chunk (gfx950).
#pragma once

#include "delta_chunk.hpp"

namespace spk {
namespace delta {

constexpr int LDS_BYTES = 160 * 1024;

// What the operand kernel leaves for the others, per (sequence, key head, chunk)
// the fragments of K and Q, and per (sequence, value head, chunk), in bytes:
//   forward   T, coefficients, P
//   backward  T, coefficients, T^T, P^T
template <class E, int DS, bool BWD>
struct Blob : Lay<E, DS> {
    using B = Lay<E, DS>;
    static constexpr int KEY = 2 * B::K;
    static constexpr int T = B::TRI * 3 * FRAG, P = T;
    static constexpr int TTAT = T + B::COEF, PAT = TTAT + (BWD ? T : 0);
    static constexpr int HEAD = PAT + P;
};

struct Chunks {
    int NC;               // chunks of the longest sequence
    char *key, *head;     // workspace
};

// What the passes over the chunks keep for the gradients, columns padded to dvp
// (a multiple of 32) and rows to whole chunks and groups of 32 of dk, in blocks of
// 16 rows and 32 columns:
//   S, dS  [b * Hv + h][chunk][2 DS][dvp / 32]  state that enters the chunk, gradient of the one that leaves it
//   U, Y   [b * Hv + h][chunk][MT][dvp / 32]
// A block is in the order in which the gradients' waves take it up as an operand:
// columns 8g..8g+3 of row i for lane (i, g), then columns 8g+4..8g+7.  (From rows of
// dvp floats a load gathers 16 rows, a cache line for each 16 bytes.)
constexpr int KEPT_BLOCK = 128;  // in f32x4
struct Kept {
    int dvp;
    f32x4 *S, *dS, *U, *Y;
};

// Result tile to block: lane (n, g) holds rows 4g..4g+3 of column n, and gets row
// 4g + n % 4 of the columns 4 (n / 4)... of its quad.
__device__ __forceinline__ f32x4 quad_transpose(f32x4 a, int lane) {
    auto swap = [&](float &lo, float &hi, bool up, auto ctrl) {  // hi of the lower lane and lo of the upper one change places
        const int x = __float_as_int(up ? lo : hi);
        const float y = __int_as_float(__builtin_amdgcn_update_dpp(x, x, decltype(ctrl)::value, 0xF, 0xF, true));
        lo = up ? y : lo;
        hi = up ? hi : y;
    };
    float x[4] = {a[0], a[1], a[2], a[3]};
    const std::integral_constant<int, 0xB1> by1;  // quad lanes 1 0 3 2
    const std::integral_constant<int, 0x4E> by2;  // quad lanes 2 3 0 1
    swap(x[0], x[1], lane & 1, by1);
    swap(x[2], x[3], lane & 1, by1);
    swap(x[0], x[2], lane & 2, by2);
    swap(x[1], x[3], lane & 2, by2);
    return (f32x4){x[0], x[1], x[2], x[3]};
}
// the lane's place in a block for a result tile of columns 16 ct.. (bytes)
__device__ __forceinline__ uint32_t block_place(int ct, int lane) {
    const int n = lane & 15, g = lane >> 4;
    return ((n >> 2) & 1) * 1024 + (2 * (ct & 1) + (n >> 3)) * 256 + (4 * g + (n & 3)) * 16;
}

// Eight elements of a row of keys or queries from 32 s + 8 g on, in the row's own
// type.  Indices past the row are clamped and the elements set to 0 afterwards:
// loads behind a branch would each be waited for.
template <class E>
struct Raw8 {
    E e[8];
};
template <class E, bool WIDE>
__device__ __forceinline__ Raw8<E> load8(const E *p, int s, int g, int dk) {
    Raw8<E> r;
    const int c = 32 * s + 8 * g;
    if constexpr (WIDE) {  // dk a multiple of 8, rows on 16 bytes
        struct alignas(16) Eight {
            E e[8];
        };
        const Eight w = *reinterpret_cast<const Eight *>(p + min(c, dk - 8));
#pragma unroll
        for (int j = 0; j < 8; ++j) r.e[j] = w.e[j];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) r.e[j] = p[min(c + j, dk - 1)];
    }
    return r;
}
template <class E>
__device__ __forceinline__ void as_floats(const Raw8<E> &w, int s, int g, int dk, bool row, float (&x)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = row && 32 * s + 8 * g + j < dk ? to_float(w.e[j]) : 0.0f;
}

// Has x computed here, before the loads that follow: their registers can then be
// those of the values that x was made from.  Made later, x would keep these alive,
// and the new ones would be waited for at once to be moved into their place.
__device__ __forceinline__ void made(float &x) { asm volatile("" : "+v"(x) : : "memory"); }

constexpr int PREP_THREADS = 256;

// Log decays above 0 may add up to this in a chunk.  A and P hold e^{gamma_i - gamma_j},
// and T and the sums over a chunk cancel what these grow by where the rule itself
// replaces it: their errors are the rule's times e to that sum (unit keys that repeat,
// beta = 1, g = 1/4: no digit is left of 64 samples).  Beyond, the chunk's
// decays become NaN, and with them all that the rule makes from it.
constexpr float MAX_RISE = 1.0f;

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
// once the products are made (and, before T, P).
template <class E, int DS>
struct PrepLds {
    using B = Lay<E, DS>;
    static constexpr int PITCH = B::C + 4;  // floats; 16-byte rows, four banks on from row to row
    static constexpr int SQ = B::C * PITCH * 4;
    static constexpr int R0 = 2 * B::K > 2 * SQ ? 2 * B::K : 2 * SQ;
    static constexpr int HEADS = PREP_THREADS / 64;  // whose decays are made at a time
    static constexpr int BYTES = R0 + HEADS * B::C * 12;
};

// Grid (chunk, b * Hk + key head): the fragments of the chunk's keys and
// queries, their products, and for each value head of the key head T, P and the
// coefficients.  The products stay in registers, a row of tiles a wave.  T by
// blocks of 16: the diagonal ones by substitution, a column a lane; the rest of
// block column j by
//     T_ij = -T_ii sum over j <= m < i of A_im T_mj
// on the float matrix cores, a block column a wave.  The steps are short and
// wait for each other, so the LDS is kept small enough for four workgroups a CU
// (dk <= 128, bfloat16).  4 x 4096 samples of 16 keys for 32 heads of 128x128,
// bfloat16: 159 us, 3.7 TB/s read and written (40 us more with the products in LDS).
template <class E, int DS, bool BWD>
__global__ __launch_bounds__(PREP_THREADS, 4) void k_delta_prep(const E *__restrict__ q, const E *__restrict__ k,
                                                                const float *__restrict__ g,
                                                                const float *__restrict__ beta, Args a,
                                                                const int32_t *__restrict__ lengths, int wide, Chunks w) {
    using F = Blob<E, DS, BWD>;
    using S = PrepLds<E, DS>;
    constexpr int C = F::C, MT = F::MT, NT = F::NT, PITCH = S::PITCH;
    extern __shared__ char lds[];
    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, gr = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int chunk = blockIdx.x, b = blockIdx.y / a.Hk, hk = blockIdx.y % a.Hk, rep = a.Hv / a.Hk;
    const int n = (lengths ? max(0, min(a.L, lengths[b])) : a.L) - chunk * C;  // samples from the chunk's first on
    if (n <= 0) return;
    char *fk = lds, *fq = lds + F::K;
    float *A = reinterpret_cast<float *>(lds), *T = A + C * PITCH;
    double *gam = reinterpret_cast<double *>(lds + S::R0);      // [HEADS][C]
    float *bet = reinterpret_cast<float *>(gam + S::HEADS * C);  // [HEADS][C]
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
                const Terms<NT> t = split<NT, true>(y);
                const int o = (mt * DS + s) * NT * FRAG;
                put_frag<NT>((isq ? fq : fk) + o, lane, t);
                put_frag<NT>(key + (isq ? F::K : 0) + o, lane, t);
            }
        }
    };
    if (wide) units(std::true_type{});
    else units(std::false_type{});
    __syncthreads();
    // lower tiles of K K^T (row wv) and Q K^T (row 3 - wv), where there are such rows
    const int grow = wv, hrow = 3 - wv;
    f32x4 G[MT], H[MT];
#pragma unroll
    for (int nt = 0; nt < MT; ++nt) {
        G[nt] = H[nt] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            if (nt <= grow && grow < MT)
                mma<NT, NT>(G[nt], frag<NT>(fk + (grow * DS + s) * NT * FRAG, lane),
                            frag<NT>(fk + (nt * DS + s) * NT * FRAG, lane));
            if (nt <= hrow && hrow < MT)
                mma<NT, NT>(H[nt], frag<NT>(fq + (hrow * DS + s) * NT * FRAG, lane),
                            frag<NT>(fk + (nt * DS + s) * NT * FRAG, lane));
        }
    }
    for (int hr = 0; hr < rep; ++hr) {
        const int hs = hr % S::HEADS;
        char *head = w.head + (((int64_t)b * a.Hv + hk * rep + hr) * w.NC + chunk) * F::HEAD;
        if (hs == 0) {  // the decays of the next heads, one a wave
            const int h = hk * rep + hr + wv;
            if (hr + wv < rep) {
                const int64_t at = ((int64_t)b * a.L + chunk * C + min(lane, n - 1)) * a.Hv + h;
                const bool in = lane < C && lane < n;
                const float gv = g[at], bv = beta[at];
                double s = in ? log_decay(gv) : 0.0;
#pragma unroll
                for (int o = 1; o < C; o <<= 1) {
                    const double p = __shfl_up(s, o, 64);
                    if (lane >= o) s += p;
                }
                float rise = in && gv > 0.0f ? gv : 0.0f;
                if (__ballot(rise > 0.0f)) {  // (uniform, and rare)
#pragma unroll
                    for (int o = 32; o >= 1; o >>= 1) rise += __shfl_xor(rise, o, 64);
                    if (rise > MAX_RISE) s = NAN;
                }
                const double end = __shfl(s, C - 1, 64);
                if (lane < C) {
                    gam[wv * C + lane] = s;
                    bet[wv * C + lane] = in ? bv : 0.0f;
                    float *co = reinterpret_cast<float *>(w.head + (((int64_t)b * a.Hv + h) * w.NC + chunk) * F::HEAD + F::T);
                    const float e = expf((float)s);
                    co[lane] = e;
                    co[C + lane] = in ? bv : 0.0f;
                    co[2 * C + lane] = expf((float)(end - s));
                    co[3 * C + lane] = a.scale * e;
                }
            }
        }
        __syncthreads();  // (the fragments', or the last head's, room is free)
        const double *gm = gam + hs * C;
        const float *bt = bet + hs * C;
        // A, and P in T's room
#pragma unroll
        for (int nt = 0; nt < MT; ++nt) {
            const int j = 16 * nt + m;
            const double gj = gm[j];
            if (nt <= grow && grow < MT) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * grow + 4 * gr + r;
                    A[i * PITCH + j] = bt[i] * expf((float)(j < i ? gm[i] - gj : 0.0)) * G[nt][r];
                }
            }
            if (nt <= hrow && hrow < MT) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * hrow + 4 * gr + r;
                    T[i * PITCH + j] = j <= i ? a.scale * expf((float)(j < i ? gm[i] - gj : 0.0)) * H[nt][r] : 0.0f;
                }
            }
        }
        __syncthreads();
        for (int u = tid; u < F::TRI * 64; u += PREP_THREADS) {  // P, or P^T
            const int f = u >> 6;
            int mt, gp;
            tri_at<MT, BWD>(f, &mt, &gp);
            const int i = 16 * mt + m;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 32 * gp + slot(gr, j), lo = BWD ? i : c, hi = BWD ? c : i;
                const float p = T[hi * PITCH + lo];
                x[j] = lo <= hi ? p : 0.0f;
            }
            put_frag<3>(head + F::PAT + f * 3 * FRAG, lane, split<3, true>(x));
        }
        float x[16];
        if (wv < MT) {  // diagonal block wv, column m (all lane groups alike)
            const float *Ab = A + 16 * wv * PITCH + 16 * wv;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                float s = i == m ? 1.0f : 0.0f;
#pragma unroll
                for (int j = 0; j < i; ++j) s -= Ab[i * PITCH + j] * x[j];
                x[i] = s;
            }
        }
        __syncthreads();
        if (wv < MT && gr == 0) {
#pragma unroll
            for (int i = 0; i < 16; ++i) T[(16 * wv + i) * PITCH + 16 * wv + m] = x[i];
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
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int c = 32 * gp + slot(gr, j), lo = up ? i : c, hi = up ? c : i;
                const float t = T[hi * PITCH + lo];
                y[j] = lo <= hi ? t : 0.0f;
            }
            put_frag<3>(head + (up ? F::TTAT : 0) + f * 3 * FRAG, lane, split<3, true>(y));
        }
        if (hr + 1 < rep) __syncthreads();
    }
}

// Workgroups go to the eight XCDs in turn; this order puts the value heads of a
// key head, which read the same operands, on one XCD's L2.
__device__ __forceinline__ int head_of(int x, int n) { return n % 8 == 0 ? (x & 7) * (n >> 3) + (x >> 3) : x; }

// Waves of a workgroup that only copy the next chunk's operands to LDS: a wave that
// issues copies waits while they go out.  1024 samples of 16 memories of 128x128, float:
// 79 us with two such waves, 73 with four or eight; 4 x 4096 samples of 32, bfloat16:
// 442 us with two or four, 994 with eight, whose registers the other waves lack.
constexpr int COPIERS = 4;

// Waves that carry columns, at most: those of one kernel are limited by their
// registers.
template <int DS, int KS>
constexpr int carriers() {
    return DS == 8 && KS == 1 ? 4 : 8;
}

// LDS of the states' kernel, for KS waves to a tile of 16 columns.  K is needed all
// through a chunk and has two buffers where they fit; T, the coefficients and P from
// the middle on, with two where those still fit; Q is done with in the middle and
// has one, or none (DIRECT) where K's second, or even its first, only fits without it
// and a wave has registers for its own part of Q.  Then the partial sums that the waves
// of a tile exchange.
template <class E, int DS, int KS, bool STATES>
struct ScanLds {
    using F = Blob<E, DS, STATES>;
    static constexpr int TP = STATES ? F::T + F::COEF : F::HEAD, TILES = carriers<DS, KS>() / KS;
    static constexpr int X = KS > 1 ? carriers<DS, KS>() * F::MT * FRAG : 0;
    static constexpr int Y = STATES ? 0 : TILES * F::MT * (KS - 1) * FRAG;
    static constexpr bool DIRECT = !STATES && F::MT * (DS / KS) * F::NT <= 12 && 3 * F::K + TP + X + Y > LDS_BYTES;
    static constexpr int Q = STATES || DIRECT ? 0 : F::K;
    static constexpr int KB = 2 * F::K + Q + TP + X + Y <= LDS_BYTES ? 2 : 1;
    static constexpr int TB = KB * F::K + Q + 2 * TP + X + Y <= LDS_BYTES ? 2 : 1;
    static constexpr int AT_Q = KB * F::K, AT_TP = AT_Q + Q, AT_X = AT_TP + TB * TP, AT_Y = AT_X + X,
                         BYTES = AT_Y + Y;
    static_assert(BYTES <= LDS_BYTES, "LDS");
};

// Grid (b * Hv + value head, block of columns): KS waves carry 16 columns of the
// state through the chunks, each the rows of its DS / KS groups of 32 of dk, in
// registers: as the right operand of K S and Q S (three terms) and as the sums of
// K^T (last U).  They add up K S through LDS in the middle of a chunk, after
// which each has U for itself; of out each finishes some rows.  KS = 1 where the
// columns alone fill the SIMDs, more where they do not.  STATES: for the backward
// pass, the state that enters each chunk and U are written instead of out (`kept`).
// The chunks of a head follow each other: bound by a chunk's chain of products,
// splits and two exchanges, 2.5 us for 32 samples of 250x10 memories, float (1000
// samples 80 us), 4.7 us for 64 of 128x128, bfloat16 (4 x 4096 samples of 32 heads
// 298 us, 173 TFLOP/s of the definition's products; the matrix cores are busy a third
// of the time).
template <class E, int DS, int KS, bool STATES>
__global__ __launch_bounds__(64 * (carriers<DS, KS>() + COPIERS)) void k_delta_scan(const E *__restrict__ v, Args a,
                                                    const int32_t *__restrict__ lengths, int tiles, Chunks w,
                                                    const float *state_in, E *__restrict__ out, float *state_out,
                                                    Kept kept) {
    using F = Blob<E, DS, STATES>;
    using M = ScanLds<E, DS, KS, STATES>;
    constexpr int C = F::C, MT = F::MT, NT = F::NT, GP = F::GP, DW = DS / KS;
    // Fragments in flight to the matrix cores.  A wave of up to two groups of dk has
    // little else to do meanwhile (2048 samples of 8 memories of 128x64, bfloat16: 103 us,
    // 108 with none); one of four, or that holds its part of Q, has no registers for them
    // (4 x 4096 samples of 32 of 128x128: 490 us, 442 with none; 1024 of 16 of 256x256:
    // 140 and 97).
    constexpr bool ROOM = DW <= 2 && !M::DIRECT;
    constexpr int AHEAD = !ROOM ? 0 : NT == 1 ? 3 : 1, AHEAD3 = ROOM ? 1 : 0;  // (of three terms)
    extern __shared__ char lds[];
    const int tid = threadIdx.x, lane = tid & 63, m = lane & 15, gr = lane >> 4;
    const int wv = __builtin_amdgcn_readfirstlane(tid >> 6), cw = wv - tiles * KS;  // cw >= 0: a copier
    const int tile = wv / KS, part = wv % KS, s0 = part * DW;  // the wave's columns and groups of dk
    const int bh = head_of(blockIdx.x, gridDim.x), b = bh / a.Hv, h = bh % a.Hv, hk = h / (a.Hv / a.Hk);
    const int n = lengths ? max(0, min(a.L, lengths[b])) : a.L, nc = (n + C - 1) / C;
    const int col = ((int)blockIdx.y * tiles + tile) * 16 + m;
    const bool mine = tile < tiles && col - m < (STATES ? kept.dvp : a.dv), live = mine && col < a.dv;
    const char *key = w.key + ((int64_t)b * a.Hk + hk) * w.NC * F::KEY;
    const char *head = w.head + (int64_t)bh * w.NC * F::HEAD;
    f32x4 S[2 * DW];
#pragma unroll
    for (int t = 0; t < 2 * DW; ++t) S[t] = (f32x4){0.f, 0.f, 0.f, 0.f};
    if (state_in) {
        const float *from = state_in + (int64_t)bh * a.dk * a.dv + min(col, a.dv - 1);
#pragma unroll
        for (int t = 0; t < 2 * DW; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = from[(int64_t)min(dk_of(2 * s0 + t, 4 * gr + r), a.dk - 1) * a.dv];
#pragma unroll
        for (int t = 0; t < 2 * DW; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) S[t][r] = live && dk_of(2 * s0 + t, 4 * gr + r) < a.dk ? S[t][r] : 0.0f;
    }
    auto fetch_k = [&](int c) { to_lds(lds + (c % M::KB) * F::K, key + (int64_t)c * F::KEY, F::K, cw, COPIERS, lane); };
    auto fetch_q = [&](int c) {
        if (M::Q) to_lds(lds + M::AT_Q, key + (int64_t)c * F::KEY + F::K, F::K, cw, COPIERS, lane);
    };
    auto fetch_t = [&](int c) {
        to_lds(lds + M::AT_TP + (c % M::TB) * M::TP, head + (int64_t)c * F::HEAD, M::TP, cw, COPIERS, lane);
    };
    // sample i of the chunk, column col: uniform rows and the lane's offset within four of them
    const int64_t vstep = (int64_t)a.Hv * a.dv;
    const E *vrow = v + ((int64_t)b * a.L * a.Hv + h) * a.dv;
    E *orow = out + ((int64_t)b * a.L * a.Hv + h) * a.dv;
    const uint32_t lin = (uint32_t)((4 * gr * vstep + min(col, a.dv - 1)) * sizeof(E)),
                   lout = (uint32_t)((4 * gr * vstep + col) * sizeof(E));
    const int ct = (int)blockIdx.y * tiles + tile, vgs = kept.dvp / 32;
    const uint32_t lkept = block_place(ct, lane);
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
    Terms<NT> qd[M::DIRECT ? DW : 1][MT];  // the wave's part of Q
    auto direct_q = [&](int c) {
        if (M::DIRECT) {
            const char *p = key + (int64_t)c * F::KEY + F::K;
#pragma unroll
            for (int s = 0; s < (M::DIRECT ? DW : 0); ++s)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) qd[s][mt] = frag<NT>(p + (mt * DS + s0 + s) * NT * FRAG, lane);
        }
    };
    auto arrived = [&] {  // what the copiers have asked for; the others' loads are waited for where they are used
        if (cw >= 0) wait_copies();
    };
    if (nc) {
        if (cw >= 0) {
            fetch_k(0);
            fetch_q(0);
            fetch_t(0);
        } else {
            values(0);
            direct_q(0);
        }
        arrived();
    }
    __syncthreads();
    for (int c = 0; c < nc; ++c) {
        const char *K = lds + (c % M::KB) * F::K, *Q = lds + M::AT_Q, *T = lds + M::AT_TP + (c % M::TB) * M::TP,
                   *P = T + F::PAT;
        const float *co = reinterpret_cast<const float *>(T + F::T);
        f32x4 X[MT], Y[MT];
        float vc[MT][4];
        if (mine) {
            if (STATES) {
                f32x4 *dst = kept.S + ((((int64_t)bh * w.NC + c) * 2 * DS + 2 * s0) * vgs + (ct >> 1)) * KEPT_BLOCK;
#pragma unroll
                for (int t = 0; t < 2 * DW; ++t) at(dst + t * vgs * KEPT_BLOCK, lkept) = quad_transpose(S[t], lane);
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) X[mt] = Y[mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
            constexpr int KQ = STATES || M::DIRECT ? 1 : 2;  // K alone, or K and Q in turn
            Terms<3> st;
            stream<DW * MT * KQ, AHEAD>(
                [&](int i) {
                    return frag<NT>((i % KQ ? Q : K) + (i / KQ % MT * DS + s0 + i / KQ / MT) * NT * FRAG, lane);
                },
                [&](int i, const Terms<NT> &f) {
                    const int s = i / KQ / MT, mt = i / KQ % MT;
                    if (i % (KQ * MT) == 0) st = split<3>(S[2 * s], S[2 * s + 1]);
                    mma<NT, 3>(i % KQ ? Y[mt] : X[mt], f, st);
                    if (M::DIRECT) mma<NT, 3>(Y[mt], qd[M::DIRECT ? s : 0][mt], st);
                });
            // the wave's own loads go out before the copies take the CU's path to memory
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    vc[mt][r] = to_float(vv[mt][r]);
                    if (STATES) vc[mt][r] = live ? vc[mt][r] : 0.0f;  // (the padding is read by others)
                    made(vc[mt][r]);
                }
            if (c + 1 < nc) {
                values(c + 1);
                direct_q(c + 1);
            }
            if (KS > 1) {
                char *xb = lds + M::AT_X + tile * KS * MT * FRAG, *yb = lds + M::AT_Y + tile * MT * (KS - 1) * FRAG;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    *reinterpret_cast<f32x4 *>(xb + (part * MT + mt) * FRAG + lane * 16) = X[mt];
                    const int own = mt * KS / MT;  // finishes these rows of out
                    if (!STATES && part != own)
                        *reinterpret_cast<f32x4 *>(yb + (mt * (KS - 1) + part - (part > own)) * FRAG + lane * 16) = Y[mt];
                }
            }
        }
        if (M::TB == 1) arrived();  // (T and P of this chunk)
        lds_barrier();
        if (c + 1 < nc && cw >= 0) {
            fetch_q(c + 1);
            if (M::KB == 2) fetch_k(c + 1);
            if (M::TB == 2) fetch_t(c + 1);
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
            f32x4 U[MT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const f32x4 ev = *reinterpret_cast<const f32x4 *>(co + 16 * mt + 4 * gr);
                const f32x4 be = *reinterpret_cast<const f32x4 *>(co + C + 16 * mt + 4 * gr);
#pragma unroll
                for (int r = 0; r < 4; ++r) X[mt][r] = be[r] * (vc[mt][r] - ev[r] * X[mt][r]);
                U[mt] = (f32x4){0.f, 0.f, 0.f, 0.f};
            }
            Terms<3> rt;
            stream<F::TRI, AHEAD3>(  // columns of 32 samples, below the diagonal
                [&](int i) { return frag<3>(T + F::lower(i < MT ? i : i - MT + 2, i < MT ? 0 : 1) * 3 * FRAG, lane); },
                [&](int i, const Terms<3> &f) {
                    const int gp = i < MT ? 0 : 1, mt = i < MT ? i : i - MT + 2;
                    if (mt == 2 * gp) rt = split<3>(X[2 * gp], X[2 * gp + 1]);
                    mma<3, 3>(U[mt], f, rt);
                });
            if (!STATES) {  // out
                const char *yb = lds + M::AT_Y + tile * MT * (KS - 1) * FRAG;
                Terms<3> ut[GP];
#pragma unroll
                for (int gp = 0; gp < GP; ++gp) ut[gp] = split<3>(U[2 * gp], U[2 * gp + 1]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    if (part != mt * KS / MT) continue;
#pragma unroll
                    for (int p = 0; p < KS - 1; ++p)
                        Y[mt] += *reinterpret_cast<const f32x4 *>(yb + (mt * (KS - 1) + p) * FRAG + lane * 16);
                    Y[mt] *= *reinterpret_cast<const f32x4 *>(co + 3 * C + 16 * mt + 4 * gr);
#pragma unroll
                    for (int gp = 0; gp <= mt / 2; ++gp)
                        mma<3, 3>(Y[mt], frag<3>(P + F::lower(mt, gp) * 3 * FRAG, lane), ut[gp]);
                }
            } else {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) Y[mt] = U[mt];
            }
            const float end = co[C - 1];  // E of the last sample
#pragma unroll
            for (int t = 0; t < 2 * DW; ++t) S[t] *= end;
            Terms<3> lt;
            stream<GP * 2 * DW, AHEAD>([&](int i) { return tfrag<NT, DS>(K, 2 * s0 + i % (2 * DW), i / (2 * DW), lane); },
                                       [&](int i, const Terms<NT> &f) {
                                           const int gp = i / (2 * DW), t = i % (2 * DW);
                                           if (t == 0) {
                                               const float *l = co + 2 * C + 32 * gp + 4 * gr;
                                               lt = split<3>(U[2 * gp] * *reinterpret_cast<const f32x4 *>(l),
                                                             U[2 * gp + 1] * *reinterpret_cast<const f32x4 *>(l + 16));
                                           }
                                           mma<NT, 3>(S[t], f, lt);
                                       });
        }
        arrived();  // the next chunk's operands
        lds_barrier();
        if (c + 1 < nc && cw >= 0) {
            if (M::KB == 1) fetch_k(c + 1);
            if (M::TB == 1) fetch_t(c + 1);
        }
        if (STATES && mine) {
            f32x4 *dst = kept.U + (((int64_t)bh * w.NC + c) * MT * vgs + (ct >> 1)) * KEPT_BLOCK;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                if (part == mt * KS / MT) at(dst + mt * vgs * KEPT_BLOCK, lkept) = quad_transpose(Y[mt], lane);
        }
        if (!STATES && live) {
            E *p = orow + (int64_t)c * C * vstep;
            const bool full = (c + 1) * C <= n;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                if (part != mt * KS / MT) continue;
                if (full) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) at(p + (16 * mt + r) * vstep, lout) = from_float<E>(Y[mt][r]);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (c * C + 16 * mt + 4 * gr + r < n) at(p + (16 * mt + r) * vstep, lout) = from_float<E>(Y[mt][r]);
                }
            }
        }
        if (M::KB == 1 && c + 1 < nc) {
            arrived();
            lds_barrier();
        }
    }
    if (!live || !state_out) return;
#pragma unroll
    for (int t = 0; t < 2 * DW; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int d = dk_of(2 * s0 + t, 4 * gr + r);
            if (d < a.dk) state_out[(int64_t)bh * a.dk * a.dv + (int64_t)d * a.dv + col] = S[t][r];
        }
}

// How a call's columns go to waves: KS waves to a tile of 16 columns and `tiles`
// of them a workgroup (`threads` in all), out of `all` tiles a head.  A CU's LDS
// takes one workgroup, so more than 256 would wait for a second turn (8 ragged
// sequences of 1531, 8 memories of 96x72, bfloat16: 111 us in 192 workgroups, 183 in 320).
// Up to there a tile's sums over dk are shared by up to eight waves, while the
// 1024 SIMDs have no more than one wave each (1000 samples of 8 memories of 250x10,
// float: 102 us with eight, 163 with one; 2 x 1024 of 16 of 256x256, bfloat16: 131
// with one, 112 with two, 128 with four), and tiles spread over more workgroups
// (2048 samples of 8 memories of 128x64, bfloat16: 126 us with two tiles each, 103
// with one).
struct Cols {
    int KS, tiles, blocks, threads;
};
inline Cols columns(const Args &a, int all, int DS) {
    Cols c;
    const int64_t heads = (int64_t)a.B * a.Hv;
    auto groups = [&](int tiles) { return heads * ((all + tiles - 1) / tiles); };
    c.KS = 1;
    while (c.KS < 8 && 2 * c.KS <= DS && heads * all * 2 * c.KS <= 1024 && groups(8 / (2 * c.KS)) <= 256) c.KS *= 2;
    const int most = (DS == 8 && c.KS == 1 ? 4 : 8) / c.KS;
    c.tiles = all < most ? all : most;
    while (c.tiles > 1 && groups((c.tiles + 1) / 2) <= 256) c.tiles = (c.tiles + 1) / 2;
    c.blocks = (all + c.tiles - 1) / c.tiles;
    c.threads = 64 * (c.tiles * c.KS + COPIERS);
    return c;
}

template <class E, int DS, int KS, bool STATES>
void launch_scan(const Cols &cols, const void *v, const Args &a, const int32_t *lengths, const Chunks &w,
                 const float *state_in, void *out, float *state_out, const Kept &kept, hipStream_t st) {
    constexpr int LDS = ScanLds<E, DS, KS, STATES>::BYTES;
    hipLaunchKernelGGL((k_delta_scan<E, DS, KS, STATES>), dim3((unsigned)(a.B * a.Hv), (unsigned)cols.blocks),
                       dim3((unsigned)cols.threads), LDS, st, static_cast<const E *>(v), a, lengths, cols.tiles, w, state_in,
                       static_cast<E *>(out), state_out, kept);
}
// CALL(KS) with the form that `cols` asks for
#define SPK_DELTA_PARTS(DS, cols, CALL)      \
    if (DS >= 8 && (cols).KS == 8) {         \
        CALL((DS >= 8 ? 8 : 1));             \
    } else if (DS >= 4 && (cols).KS == 4) {  \
        CALL((DS >= 4 ? 4 : 1));             \
    } else if (DS >= 2 && (cols).KS == 2) {  \
        CALL((DS >= 2 ? 2 : 1));             \
    } else {                                 \
        CALL(1);                             \
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

// Whether rows of dk elements can be read eight at a time.
template <class E>
int wide_rows(int dk, const void *q, const void *k) {
    return dk % 8 == 0 && aligned16(q) && aligned16(k);
}

}  // namespace delta
}  // namespace spk
