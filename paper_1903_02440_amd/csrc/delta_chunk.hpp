// The gated delta rule over chunks of C samples: what its kernels share.
//
// Within a chunk that a state S enters, with gamma the running sum of the log
// decays, E_i = e^{gamma_i}, D_ij = e^{gamma_i - gamma_j} (j <= i), and
// last_i = e^{gamma_C - gamma_i}:
//     (I + A) U = beta (V - E K S)      A_ij = beta_i D_ij k_i . k_j  (j < i)
//     out       = scale (E Q S + P U)   P_ij = D_ij q_i . k_j         (j <= i)
//     S        <- E_C S + K^T (last U)
// (P is kept times the scale.)
// T = (I + A)^-1, P and the decays depend on the inputs alone, so all chunks
// make them at once; the states then go through the chunks in order.
//
// Products run on the 16-bit matrix cores with float sums.  A float operand is
// the exact sum of three bfloat16 terms (8 bits each), a bfloat16 input is one;
// of a product of two such sums the products of terms below 2^-22 of the whole are
// left out.  Against the float matrix cores (1/16 of the rate) three or six products
// of terms cost 3/16 to 6/16, at the same precision.
//
// Operands lie in fragments: for 16 rows and 32 summed indices the 16 bytes of
// each lane in turn (1 KiB a term).  The result of a matrix instruction holds,
// in lane (n, g), rows 4g..4g+3 of column n; two result tiles taken as one right
// operand give lane group g eight of the 32 indices.  The left operands are laid
// out for that order, so results feed the next product without leaving their
// lane: samples go by slot() below, and the rows of the state's tiles are dealt
// out by dk_of() so that lane group g holds 8g..8g+7, as a row of K lies in
// memory.  K^T is read from the fragments of K by the LDS's transposing reads.
#pragma once

#include <type_traits>

#include "delta.hpp"

namespace spk {
namespace delta {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int FRAG = 1024;  // bytes of one term of a fragment

// index within a group of 32 samples (or columns) of element j of lane group g
__device__ __forceinline__ int slot(int g, int j) { return j < 4 ? 4 * g + j : 12 + 4 * g + j; }

// index in dk of row i of the state's tile t
__device__ __forceinline__ int dk_of(int t, int i) { return 32 * (t >> 1) + 8 * (i >> 2) + 4 * (t & 1) + (i & 3); }

template <int N>
struct Terms {
    u32x4 t[N];
};

// The upper halves of two floats as one word.
__device__ __forceinline__ uint32_t upper2(uint32_t lo, uint32_t hi) {
    return __builtin_amdgcn_perm(hi, lo, 0x07060302u);
}

// Eight floats as N bfloat16 terms: three hold every float.  Cut off, each term
// takes the leading 8 bits of what is left; NEAREST, the first two are rounded, and
// may have the other sign.  One operand of a product is to be NEAREST: the products
// that mma() leaves out, of second and third terms, are then below 2^-22 of the whole,
// without a preferred sign.  (Of two operands that are cut off it would be 2^-21, always
// below the true product.)  It is the one made outside the passes over the chunks,
// which are 2 to 5 % slower where they round.  A single term is rounded.
template <int N, bool NEAREST = false>
__device__ __forceinline__ Terms<N> split(const float (&x)[8]) {
    constexpr float MOST = 3.38953139e38f;  // the largest bfloat16: rounding is not to reach infinity
    Terms<N> r;
    float y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = x[j];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bool nearest = N == 1 || (NEAREST && i < 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool clamp = NEAREST && N == 3 && i == 0;
            const float lo = clamp ? __builtin_amdgcn_fmed3f(y[2 * j], -MOST, MOST) : y[2 * j];
            const float hi = clamp ? __builtin_amdgcn_fmed3f(y[2 * j + 1], -MOST, MOST) : y[2 * j + 1];
            r.t[i][j] = nearest ? (uint32_t)from_float<uint16_t>(lo) | ((uint32_t)from_float<uint16_t>(hi) << 16)
                                : upper2(__float_as_uint(lo), __float_as_uint(hi));
        }
        if (i == N - 1) break;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t w = nearest ? r.t[i][j >> 1] : __float_as_uint(y[j]);
            y[j] -= __uint_as_float(nearest && !(j & 1) ? w << 16 : w & 0xFFFF0000u);
        }
    }
    return r;
}
template <int N>
__device__ __forceinline__ Terms<N> split(const f32x4 &a, const f32x4 &b) {
    const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
    return split<N>(x);
}

__device__ __forceinline__ f32x4 mfma(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
                                                   0, 0);
}

// c += a b, smaller products of terms first.
template <int NA, int NB>
__device__ __forceinline__ void mma(f32x4 &c, const Terms<NA> &a, const Terms<NB> &b) {
    constexpr int M = NA > NB ? NA : NB;
#pragma unroll
    for (int o = M - 1; o >= 0; --o)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (o - i >= 0 && o - i < NB) c = mfma(a.t[i], b.t[o - i], c);
}

// Element at a uniform place p plus the lane's own 32-bit byte offset: the
// address costs no vector instruction.
template <class T>
__device__ __forceinline__ T &at(T *p, uint32_t bytes) {
    using Byte = typename std::conditional<std::is_const<T>::value, const char, char>::type;
    return *reinterpret_cast<T *>(reinterpret_cast<Byte *>(p) + bytes);
}

// The lane's part of a fragment of N terms.
template <int N>
__device__ __forceinline__ Terms<N> frag(const char *p, int lane) {
    Terms<N> r;
#pragma unroll
    for (int i = 0; i < N; ++i) r.t[i] = *reinterpret_cast<const u32x4 *>(p + i * FRAG + lane * 16);
    return r;
}
template <int N>
__device__ __forceinline__ void put_frag(char *p, int lane, const Terms<N> &x) {
#pragma unroll
    for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4 *>(p + i * FRAG + lane * 16) = x.t[i];
}

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Fragment of the transpose of K (or Q) in LDS: rows of the state's tile t,
// samples of group gp.  A transposing read gives lane i of a group of 16 the
// i-th column of four rows of 16, here four samples' values of dk_of(t, i).
template <int NT, int DS>
__device__ __forceinline__ Terms<NT> tfrag(const char *k, int t, int gp, int lane) {
    const int i = lane & 15, g = lane >> 4;
    Terms<NT> r;
#pragma unroll
    for (int x = 0; x < NT; ++x)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
            const char *p = k + (((2 * gp + hf) * DS + (t >> 1)) * NT + x) * FRAG + ((i & 3) * 16 + 4 * g + (i >> 2)) * 16 +
                            8 * (t & 1);
            const s16x4 w = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) s16x4 *)const_cast<char *>(p));
            const uint2 u = __builtin_bit_cast(uint2, w);
            r.t[x][2 * hf] = u.x, r.t[x][2 * hf + 1] = u.y;
        }
    return r;
}

// use(i, load(i)) for i < N, with the loads AHEAD items before their use (0: where
// the compiler likes, which is right before the products that wait for them).
template <int N, int AHEAD, class Load, class Use>
__device__ __forceinline__ void stream(Load load, Use use) {
    decltype(load(0)) f[AHEAD + 1];
#pragma unroll
    for (int i = 0; i < AHEAD && i < N; ++i) f[i] = load(i);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i + AHEAD < N) f[(i + AHEAD) % (AHEAD + 1)] = load(i + AHEAD);
        if (AHEAD) asm volatile("" ::: "memory");
        use(i, f[i % (AHEAD + 1)]);
    }
}

// Sizes of a chunk's operands.  DS: groups of 32 of dk; MT: tiles of 16
// samples.  Float inputs take chunks of 32 samples, so that their three terms
// fit the LDS at dk = 256; bfloat16 ones take 64.
template <class E>
struct Type;
template <>
struct Type<float> {
    static constexpr int NT = 3, MT = 2;
};
template <>
struct Type<uint16_t> {
    static constexpr int NT = 1, MT = 4;
};
template <class E, int DS>
struct Lay {
    static constexpr int NT = Type<E>::NT, MT = Type<E>::MT;
    static constexpr int C = 16 * MT, GP = MT / 2;
    // a triangular C x C operand: the fragments that are not zero throughout
    static constexpr int TRI = MT == 4 ? 6 : 2;
    static constexpr int K = MT * DS * NT * FRAG;  // rows of K (or Q), summed over dk: [mt][s][term]
    static constexpr int COEF = FRAG;              // E, beta, last, scale E: f32 [4][C]
    // fragment (mt, gp <= mt / 2) of a lower triangular operand
    static __host__ __device__ constexpr int lower(int mt, int gp) { return mt < 2 ? mt : 2 * mt - 2 + gp; }
    // fragment (mt, gp >= mt / 2) of an upper triangular one
    static __host__ __device__ constexpr int upper(int mt, int gp) {
        return MT == 2 ? mt : mt < 2 ? 2 * mt + gp : mt + 2;
    }
};

constexpr int chunk_of(int dtype) { return dtype == SPK_F32 ? 32 : 64; }

// e^g for sums of log decays: -inf (all forgotten) as a number whose
// exponential is 0, so that differences of sums stay defined.
__device__ __forceinline__ double log_decay(float g) { return g < -1e4f ? -1e4 : (double)g; }

// Copies n bytes (a multiple of 1 KiB) to LDS past the registers; both ends
// 16-byte aligned.  All waves of the workgroup take part.  The copy is one the
// compiler does not count: before use, wait for vmcnt(0) and then a barrier.
// (As a builtin it would make every LDS read wait for it, also those of another
// buffer.)  The wait state that a copy needs after a write of m0 is in the statement:
// the compiler adds none for an instruction of inline assembly.
__device__ __forceinline__ void to_lds(char *dst, const char *src, int n, int wave, int waves, int lane) {
    const uint32_t at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)dst;
    for (int o = wave * FRAG; o < n; o += waves * FRAG)
        asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src + o + lane * 16),
                     "{m0}"(__builtin_amdgcn_readfirstlane((int)(at + o)))
                     : "memory");
}
// A barrier that hands LDS over; copies and loads may stay in flight.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
// All of the wave's copies and loads have arrived, its stores are out.  (As a
// builtin the compiler counts it too: loads before it need no wait of their own.)
__device__ __forceinline__ void wait_copies() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);  // vmcnt(0)
    asm volatile("" ::: "memory");
}

}  // namespace delta
}  // namespace spk
