// Gated delta rule of a linear readout (gfx950): one sample after another.
//
//     u_t   = beta_t (v_t - a_t S^T k_t)       a_t = e^{g_t}, S the state before sample t
//     S_t   = a_t S + k_t u_t^T
//     out_t = scale S_t^T q_t = scale (a_t S^T q_t + (k_t . q_t) u_t)
//
// Columns of S are independent of each other, rows meet in two sums over dk.
#include <cmath>
#include <type_traits>

#include "delta.hpp"

namespace spk {
namespace delta {

int check(const Args &a, const char *name) {
    SPK_REQUIRE(a.dtype == SPK_F32 || a.dtype == SPK_BF16, SPK_E_ARG, "%s: dtype %d is neither SPK_F32 nor SPK_BF16",
                name, a.dtype);
    SPK_REQUIRE(a.B >= 0 && a.L >= 0 && a.Hk >= 1 && a.Hv >= 1 && a.dk >= 1 && a.dv >= 1, SPK_E_SHAPE, "%s: bad sizes",
                name);
    SPK_REQUIRE(a.Hv % a.Hk == 0, SPK_E_SHAPE, "%s: Hv=%d is not a multiple of Hk=%d", name, a.Hv, a.Hk);
    SPK_REQUIRE(a.dk <= 256, SPK_E_RANGE, "%s: dk=%d > 256", name, a.dk);
    SPK_REQUIRE(a.dv <= 4096, SPK_E_RANGE, "%s: dv=%d > 4096", name, a.dv);
    SPK_REQUIRE((int64_t)a.B * a.Hv <= 65535, SPK_E_RANGE, "%s: B*Hv above 65535", name);
    SPK_REQUIRE((int64_t)a.Hv * a.dv <= (1 << 22), SPK_E_RANGE, "%s: Hv*dv above 2^22", name);
    SPK_REQUIRE(a.L <= (1 << 24), SPK_E_RANGE, "%s: L=%d > 2^24", name, a.L);
    SPK_REQUIRE(std::isfinite(a.scale), SPK_E_ARG, "%s: scale must be finite", name);
    return SPK_OK;
}

}  // namespace delta
}  // namespace spk

using namespace spk::delta;

namespace {

constexpr int THREADS = 256;

// VW neighbouring floats on any float's place
typedef float float4u __attribute__((ext_vector_type(4), aligned(4)));
typedef float float1u __attribute__((ext_vector_type(1), aligned(4)));
template <int VW>
using Cols = typename std::conditional<VW == 4, float4u, float1u>::type;

// Grid (b * Hv + h, column block).  A thread holds RT rows of VW neighbouring
// columns of S in registers: lanes run over CL = 2^cl column groups first, then
// over row groups, so that a row of S is read and written in one run.  Where dv is
// no multiple of four, the last group of columns starts earlier to stay inside its
// row, and writes only the columns that are its own.  Both sums over dk go through
// the wave's shuffles and then LDS, with one barrier a sample (the LDS sums
// alternate between two buffers).  One sample is bound by reading and writing the
// states: 256 x 32 of 128x128 in 230 us, 4.7 TB/s (a copy reaches 4.9).
template <class E, int VW, int RT>
__global__ __launch_bounds__(THREADS) void k_delta_seq(const E *__restrict__ q, const E *__restrict__ k,
                                                       const E *__restrict__ v, const float *__restrict__ g,
                                                       const float *__restrict__ beta, Args a, int cl,
                                                       const int32_t *__restrict__ lengths, const float *state_in,
                                                       E *__restrict__ out, float *state_out) {
    __shared__ float red[2][THREADS / 64][64 * VW * 2 + 1];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const int CL = 1 << cl, RG = THREADS >> cl;
    const int cg = ((int)blockIdx.y * CL + (tid & (CL - 1))) * VW, rg = tid >> cl;  // first column of its own
    const bool in = cg < a.dv;
    const int c0 = min(cg, a.dv - VW);
    const int b = blockIdx.x / a.Hv, h = blockIdx.x % a.Hv, hk = h / (a.Hv / a.Hk);
    const int n = lengths ? max(0, min(a.L, lengths[b])) : a.L;
    const int64_t s0 = (int64_t)blockIdx.x * a.dk * a.dv;
    float S[RT][VW];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < VW; ++j) S[i][j] = 0.0f;
    if (state_in) {
        Cols<VW> w[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i)
            w[i] = *reinterpret_cast<const Cols<VW> *>(state_in + s0 + (int64_t)min(rg + i * RG, a.dk - 1) * a.dv + c0);
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int j = 0; j < VW; ++j) S[i][j] = rg + i * RG < a.dk ? w[i][j] : 0.0f;
    }
    for (int t = 0; t < n; ++t) {
        const int64_t row = (int64_t)b * a.L + t;
        const E *kp = k + (row * a.Hk + hk) * a.dk, *qp = q + (row * a.Hk + hk) * a.dk;
        const float al = expf(g[row * a.Hv + h]), be = beta[row * a.Hv + h];
        float kr[RT], sk[VW], sq[VW], kq = 0.0f;
#pragma unroll
        for (int j = 0; j < VW; ++j) sk[j] = sq[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int r = rg + i * RG;
            kr[i] = r < a.dk ? to_float(kp[r]) : 0.0f;
            const float qr = r < a.dk ? to_float(qp[r]) : 0.0f;
            kq += kr[i] * qr;
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                S[i][j] *= al;
                sk[j] += S[i][j] * kr[i];
                sq[j] += S[i][j] * qr;
            }
        }
        for (int s = CL; s < 64; s <<= 1) {  // row groups of this wave
            kq += __shfl_xor(kq, s, 64);
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                sk[j] += __shfl_xor(sk[j], s, 64);
                sq[j] += __shfl_xor(sq[j], s, 64);
            }
        }
        float *mine = red[t & 1][wv];
#pragma unroll
        for (int j = 0; j < VW; ++j) {
            mine[(lane & (CL - 1)) * VW + j] = sk[j];
            mine[64 * VW + (lane & (CL - 1)) * VW + j] = sq[j];
        }
        if (lane == 0) mine[64 * VW * 2] = kq;
        __syncthreads();
        kq = 0.0f;
#pragma unroll
        for (int j = 0; j < VW; ++j) sk[j] = sq[j] = 0.0f;
        for (int w = 0; w < THREADS / 64; ++w) {
            const float *p = red[t & 1][w];
            kq += p[64 * VW * 2];
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                sk[j] += p[(lane & (CL - 1)) * VW + j];
                sq[j] += p[64 * VW + (lane & (CL - 1)) * VW + j];
            }
        }
        const int64_t o = (row * a.Hv + h) * a.dv + c0;
#pragma unroll
        for (int j = 0; j < VW; ++j) {
            const float u = be * (to_float(v[o + j]) - sk[j]);
            if (rg == 0 && in && c0 + j >= cg) out[o + j] = from_float<E>(a.scale * (sq[j] + kq * u));
#pragma unroll
            for (int i = 0; i < RT; ++i) S[i][j] += kr[i] * u;
        }
    }
    if (!state_out) return;
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        const int r = rg + i * RG;
        if (r >= a.dk || !in) continue;
        float *p = state_out + s0 + (int64_t)r * a.dv + c0;
        if (c0 == cg) {
            Cols<VW> w;
#pragma unroll
            for (int j = 0; j < VW; ++j) w[j] = S[i][j];
            *reinterpret_cast<Cols<VW> *>(p) = w;
        } else {
#pragma unroll
            for (int j = 0; j < VW; ++j)
                if (c0 + j >= cg) p[j] = S[i][j];
        }
    }
}

template <class E>
void launch_seq(const void *q, const void *k, const void *v, const float *g, const float *beta, const Args &a,
                const int32_t *lengths, const float *state_in, void *out, float *state_out, hipStream_t st) {
    const bool wide = a.dv >= 4;
    const int groups = wide ? (a.dv + 3) / 4 : a.dv;
    int cl = 0;
    while ((1 << cl) < groups && cl < 5) ++cl;
    // A row of at most 32 column groups goes in blocks of fewer where those leave an eighth
    // fewer lanes without one: 1600 of 200x77, 32 groups wide 93 us, 8 wide 71.  Longer rows
    // lose more by their shorter runs than lanes do: 8192 of 127x129, 32 wide 358 us, 8 wide 452.
    auto lanes = [&](int c) { return spk::ceil_div(groups, 1 << c) << c; };
    for (int c = cl - 1; groups <= 32 && c >= 3; --c)
        if (8 * lanes(c) <= 7 * lanes(cl)) cl = c;
    const int RG = THREADS >> cl, rt = (a.dk + RG - 1) / RG;
    const dim3 grid((unsigned)(a.B * a.Hv), (unsigned)spk::ceil_div(groups, 1 << cl));
#define SPK_SEQ(VW, RT)                                                                                              \
    hipLaunchKernelGGL((k_delta_seq<E, VW, RT>), grid, dim3(THREADS), 0, st, static_cast<const E *>(q),              \
                       static_cast<const E *>(k), static_cast<const E *>(v), g, beta, a, cl, lengths, state_in,      \
                       static_cast<E *>(out), state_out)
    if (wide) {
        if (rt <= 4) SPK_SEQ(4, 4);
        else if (rt <= 8) SPK_SEQ(4, 8);
        else if (rt <= 16) SPK_SEQ(4, 16);
        else SPK_SEQ(4, 32);
    } else {
        SPK_SEQ(1, 4);  // (at most 4 column groups: 64 rows at a time)
    }
#undef SPK_SEQ
}

// A call of more samples goes in chunks: below, two launches and a whole chunk's
// products cost more than going sample by sample.  8 x 250x10 memories, float: 15.2 us
// against 19.2 in chunks for 8 samples, 20.8 against 19.9 for 12; 512 x 128x128,
// bfloat16: 46 against 56 for 8, 56 either way for 10, 65 against 56 for 12.
bool in_chunks(const Args &a) { return a.L > 10; }

}  // namespace

extern "C" size_t spk_delta_rule_workspace_size(int dtype, int B, int L, int Hk, int Hv, int dk, int dv) {
    const Args a{dtype, B, L, Hk, Hv, dk, dv, 1.0f};
    return check(a, "") == SPK_OK && in_chunks(a) ? chunk_workspace(a) : 0;
}

extern "C" int spk_delta_rule(const void *q, const void *k, const void *v, const float *g, const float *beta, int dtype,
                              int B, int L, int Hk, int Hv, int dk, int dv, float scale, const int32_t *lengths,
                              const float *initial_state, void *out, float *final_state, void *workspace,
                              size_t ws_bytes, void *stream) {
    const char *name = "spk_delta_rule";
    const Args a{dtype, B, L, Hk, Hv, dk, dv, scale};
    if (int rc = check(a, name)) return rc;
    if (B == 0) return spk::ok();
    SPK_REQUIRE((q && k && v && g && beta && out) || L == 0, SPK_E_ARG, "%s: q, k, v, g, beta and out are required",
                name);
    if (L == 0 && !final_state) return spk::ok();
    hipStream_t st = spk::as_stream(stream);
    if (in_chunks(a)) {
        const size_t need = chunk_workspace(a);
        SPK_REQUIRE(workspace && ws_bytes >= need, SPK_E_WORKSPACE, "%s: workspace of %zu bytes, %zu needed", name,
                    workspace ? ws_bytes : (size_t)0, need);
        SPK_REQUIRE(aligned16(workspace), SPK_E_ARG, "%s: the workspace must be 16-byte aligned", name);
        return chunk_forward(q, k, v, g, beta, a, lengths, initial_state, out, final_state, workspace, st, name);
    }
    if (dtype == SPK_F32) launch_seq<float>(q, k, v, g, beta, a, lengths, initial_state, out, final_state, st);
    else launch_seq<uint16_t>(q, k, v, g, beta, a, lengths, initial_state, out, final_state, st);
    return spk::check_launch(name);
}

extern "C" int spk_delta_rule_step(const void *q, const void *k, const void *v, const float *g, const float *beta,
                                   int dtype, int B, int Hk, int Hv, int dk, int dv, float scale, float *state,
                                   void *out, void *stream) {
    const char *name = "spk_delta_rule_step";
    const Args a{dtype, B, 1, Hk, Hv, dk, dv, scale};
    if (int rc = check(a, name)) return rc;
    if (B == 0) return spk::ok();
    SPK_REQUIRE(q && k && v && g && beta && state && out, SPK_E_ARG,
                "%s: q, k, v, g, beta, state and out are required", name);
    hipStream_t st = spk::as_stream(stream);
    if (dtype == SPK_F32) launch_seq<float>(q, k, v, g, beta, a, nullptr, state, out, state, st);
    else launch_seq<uint16_t>(q, k, v, g, beta, a, nullptr, state, out, state, st);
    return spk::check_launch(name);
}
