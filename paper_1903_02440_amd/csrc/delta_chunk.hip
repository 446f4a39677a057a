// The gated delta rule over chunks of samples (gfx950): the batch call.  The
// formulas and the operands' layout are in delta_chunk.hpp, the kernels that it
// shares with the backward pass in delta_kernels.hpp.
#include "delta_kernels.hpp"

namespace spk {
namespace delta {

template <class E, int DS>
size_t carve(void *ws, const Args &a, Chunks *w) {
    using F = Blob<E, DS, false>;
    spk::Carver c(ws);
    w->NC = (a.L + F::C - 1) / F::C;
    w->key = c.take<char>((size_t)a.B * a.Hk * w->NC * F::KEY);
    w->head = c.take<char>((size_t)a.B * a.Hv * w->NC * F::HEAD);
    return spk::align_up(c.off, 256);
}

template <class E, int DS>
int forward(const void *q, const void *k, const void *v, const float *g, const float *beta, const Args &a,
            const int32_t *lengths, const float *state_in, void *out, float *state_out, void *ws, hipStream_t st,
            const char *name) {
    Chunks w;
    carve<E, DS>(ws, a, &w);
    const E *qe = static_cast<const E *>(q), *ke = static_cast<const E *>(k);
    const int wide = wide_rows<E>(a.dk, q, k);
    constexpr int LP = PrepLds<E, DS>::BYTES;
    static_assert(LP <= LDS_BYTES, "LDS");
    hipLaunchKernelGGL((k_delta_prep<E, DS, false>), dim3((unsigned)w.NC, (unsigned)(a.B * a.Hk)), dim3(PREP_THREADS), LP, st,
                       qe, ke, g, beta, a, lengths, wide, w);
    const Cols cols = columns(a, (a.dv + 15) / 16, DS);
#define SPK_SCAN(KS) launch_scan<E, DS, KS, false>(cols, v, a, lengths, w, state_in, out, state_out, Kept{}, st)
    SPK_DELTA_PARTS(DS, cols, SPK_SCAN)
#undef SPK_SCAN
    return spk::check_launch(name);
}

size_t chunk_workspace(const Args &a) {
    Chunks w;
#define SPK_WS(DS) return a.dtype == SPK_F32 ? carve<float, DS>(nullptr, a, &w) : carve<uint16_t, DS>(nullptr, a, &w)
    SPK_DELTA_FORMS(SPK_WS)
#undef SPK_WS
}

int chunk_forward(const void *q, const void *k, const void *v, const float *g, const float *beta, const Args &a,
                  const int32_t *lengths, const float *state_in, void *out, float *state_out, void *ws, hipStream_t st,
                  const char *name) {
#define SPK_FW(DS)                                                                                              \
    return a.dtype == SPK_F32                                                                                   \
               ? forward<float, DS>(q, k, v, g, beta, a, lengths, state_in, out, state_out, ws, st, name)       \
               : forward<uint16_t, DS>(q, k, v, g, beta, a, lengths, state_in, out, state_out, ws, st, name)
    SPK_DELTA_FORMS(SPK_FW)
#undef SPK_FW
}

}  // namespace delta
}  // namespace spk
