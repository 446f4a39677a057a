/*
 * libspyke_readout.h -- C ABI of the readout operators (gfx950): a readout
 * learnt from features by the gated delta rule, and winners drawn from scores
 * with given random numbers.
 *
 * The conventions of libspyke.h hold for every entry point here: device
 * pointers owned by the caller, contiguous, row-major and batch-major; scratch
 * from a caller workspace; work enqueued on `stream` without synchronising the
 * host; arguments validated on the host before anything is enqueued; SPK_E_*
 * statuses with spk_last_error().  Pointers need the alignment of their
 * element only; 16-byte aligned ones (and row lengths that are multiples of
 * 16 bytes) take wider loads.  A workspace must be 16-byte aligned, and calls
 * that may run at the same time need one each.  Outputs must not overlap inputs
 * or each other unless stated.
 */
#ifndef LIBSPYKE_READOUT_H
#define LIBSPYKE_READOUT_H

#include "libspyke.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of the `dtype` arguments. */
enum { SPK_F32 = 0, SPK_BF16 = 1 };

/* ------------------------------------------------------------------------
 * Gated delta rule: supervised plasticity of a linear readout, sample after
 * sample (ordered replay within the batch, as spk_stdp's).  Each sequence b
 * and value head h holds a weight matrix S [dk][dv]; its sample t has a key
 * k_t (features), a value v_t (what the readout should give for them), a
 * query q_t, a rate beta_t and a log decay g_t (forgetting; 0 = none):
 *     u_t   = beta_t (v_t - e^{g_t} S_{t-1}^T k_t)
 *     S_t   = e^{g_t} S_{t-1} + k_t u_t^T
 *     out_t = scale S_t^T q_t
 * so out_t is read after sample t was learnt (the next sample's key as q_t
 * gives the prediction for it before it is learnt, up to its decay).  For
 * keys of unit norm and 0 <= beta <= 1 the update contracts; longer keys or
 * larger rates can grow without bound, as the rule does.
 *   q, k       dtype [B][L][Hk][dk]; value head h reads key head h / (Hv/Hk).
 *   v, out     dtype [B][L][Hv][dv].
 *   g, beta    f32 [B][L][Hv]; g <= 0 (-inf forgets all).  A state may also
 *              grow a little: the g above 0 of any 64 samples in a row may
 *              add up to 1.  Where a call of more than 10 samples, or one for
 *              gradients, finds more it makes what depends on those samples
 *              NaN, in their sequence and head: the outputs from up to 63
 *              samples before them on, the final state, the gradients (those
 *              of q and k for the whole key head).  Up to 10 samples go one
 *              by one and take any g whose e^g is finite.
 *   lengths    i32 [B] or NULL (all L): samples of each sequence, read as
 *              clamped to [0, L].  Rows of out behind a sequence's length are
 *              not written, and input rows behind it are not read.
 *   initial_state  f32 [B][Hv][dk][dv] or NULL (zeros).
 *   final_state    f32 [B][Hv][dk][dv] or NULL (not wanted); may be
 *              initial_state (updated in place).  A sequence of no samples
 *              leaves its state as it was.
 * All sums and states are held in float; bfloat16 inputs are exact terms of
 * the products.  Repeated calls give the same bits.  Inputs up to the lengths
 * are to be finite (g may be -inf): one that is not makes outputs of its own
 * sequence and head non-finite, up to 63 samples before it too.
 * Limits: 1 <= dk <= 256, 1 <= dv <= 4096, Hv a multiple of Hk, B*Hv <= 65535,
 * Hv*dv <= 2^22, L <= 2^24.  Workspace: spk_delta_rule_workspace_size(...) bytes.          */
SPK_API size_t spk_delta_rule_workspace_size(int dtype, int B, int L, int Hk, int Hv, int dk, int dv);
SPK_API int spk_delta_rule(const void *q, const void *k, const void *v, const float *g, const float *beta, int dtype,
                           int B, int L, int Hk, int Hv, int dk, int dv, float scale, const int32_t *lengths,
                           const float *initial_state, void *out, float *final_state, void *workspace,
                           size_t ws_bytes, void *stream);

/* One sample of every sequence, the states updated in place (the online form:
 * a call per sample equals one spk_delta_rule call over them, up to rounding).
 *   q, k  dtype [B][Hk][dk]; v, out  dtype [B][Hv][dv]; g, beta  f32 [B][Hv];
 *   state f32 [B][Hv][dk][dv].
 * Limits as spk_delta_rule; any g whose e^g is finite.  No workspace.       */
SPK_API int spk_delta_rule_step(const void *q, const void *k, const void *v, const float *g, const float *beta,
                                int dtype, int B, int Hk, int Hv, int dk, int dv, float scale, float *state, void *out,
                                void *stream);

/* Gradients of spk_delta_rule's (out, final_state) with respect to all its
 * inputs, for rates, decays, keys and values that are themselves learnt.
 *   d_out          dtype [B][L][Hv][dv].
 *   d_final_state  f32 [B][Hv][dk][dv] or NULL (zeros).
 *   d_q, d_k       dtype [B][L][Hk][dk], summed over the value heads of a
 *                  key head; d_v dtype [B][L][Hv][dv]; d_g, d_beta
 *                  f32 [B][L][Hv]; all required.
 *   d_initial_state f32 [B][Hv][dk][dv] or NULL (not wanted); may be
 *                  d_final_state.
 * The other arguments are those of the forward call; its states are computed
 * again.  Rows behind a sequence's length are neither read nor written.
 * Repeated calls give the same bits.  Limits as spk_delta_rule.
 * Workspace: spk_delta_rule_backward_workspace_size(...) bytes.             */
SPK_API size_t spk_delta_rule_backward_workspace_size(int dtype, int B, int L, int Hk, int Hv, int dk, int dv);
SPK_API int spk_delta_rule_backward(const void *q, const void *k, const void *v, const float *g, const float *beta,
                                    int dtype, int B, int L, int Hk, int Hv, int dk, int dv, float scale,
                                    const int32_t *lengths, const float *initial_state, const void *d_out,
                                    const float *d_final_state, void *d_q, void *d_k, void *d_v, float *d_g,
                                    float *d_beta, float *d_initial_state, void *workspace, size_t ws_bytes,
                                    void *stream);

/* ------------------------------------------------------------------------
 * One winner per image drawn from its neurons' scores (spk_kwta with k = 1
 * takes the largest; exploration under a reward draws instead).  Among an
 * image's eligible neurons -- t_first < T (all of them when t_first is NULL),
 * score neither NaN nor -infinity -- ordered by score from largest, equal
 * scores by ascending linear index:
 *   1. the first top_k stay (0: all);
 *   2. with w = exp((score - largest) / temperature), the shortest run from
 *      the first whose w sum to at least top_p of step 1's sum stays;
 *   3. those with w >= min_p stay;
 *   4. of the rest, in ascending linear index, the winner is the first at
 *      which the running sum of w exceeds u times their sum.
 * temperature 0 takes the first of the order.  Scores of +infinity share the
 * draw among themselves.
 *   scores    dtype [B][C][H][W] (potentials of a layer whose neurons fire at
 *             one step, or class scores with H = W = 1).
 *   t_first   u8 [B][C][H][W] or NULL.
 *   u         f32 [B], uniform in [0, 1); values outside (or NaN) are taken
 *             as the nearest end (NaN: 0).
 *   winners   i32 [B][1][4] = (feature, t, y, x), t = 0 when t_first is NULL;
 *             -1 where no neuron is eligible; n_winners i32 [B], 1 or 0 (the
 *             form spk_decide and spk_rstdp read).
 * w is held as a 64-bit fixed-point number with 62 - ceil(log2(C*H*W))
 * fraction bits (51 at most), off by 1e-14 of itself and half a step at most,
 * so that sums do not depend on their order: repeated calls give the same
 * winners.
 * Limits: 0 <= temperature < inf, 0 <= top_k, 0 < top_p <= 1,
 * 0 <= min_p <= 1, 1 <= T <= 255, C*H*W <= 2^24, B <= 2^21 (65535
 * where C*H*W > 16384).
 * Workspace: spk_sample_winners_workspace_size(...) bytes.                  */
SPK_API size_t spk_sample_winners_workspace_size(int dtype, int B, int C, int H, int W);
SPK_API int spk_sample_winners(const void *scores, int dtype, const uint8_t *t_first, const float *u, int B, int T,
                               int C, int H, int W, float temperature, int top_k, float top_p, float min_p,
                               int32_t *winners, int32_t *n_winners, void *workspace, size_t ws_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* LIBSPYKE_READOUT_H */
